"""Writing tokens into the 4-bit cache and reading them back: the bytes, the
scales and the values, exactly."""
import numpy as np
import pytest
import torch

from lm_util import DEV, DT, normal, strided
from serve_util import key_bytes, rng, value_bytes, width

pytestmark = pytest.mark.gpu


def _quantized(x, pow2):
    """Codes and float32 scales of rows of float64 x."""
    big = x.abs().amax(-1)
    if pow2:
        s = torch.ldexp(torch.ones_like(big), torch.frexp(big)[1] - 3)
    else:
        s = big / 7
    s = torch.where(big > 0, s, torch.zeros_like(s)).float().clamp_min(2.0 ** -60)
    return torch.floor(x / s.double()[..., None] + 0.5).clamp(-7, 7), s


CASES = [(1, 1, 128, 16, "bf16", False), (5, 2, 64, 16, "fp32", False), (33, 3, 80, 48, "fp16", True), (70, 2, 96, 32, "bf16", True),
         (40, 1, 256, 64, "fp32", False), (17, 4, 192, 16, "bf16", False), (9, 2, 7, 16, "fp32", False), (19, 2, 36, 16, "fp16", False),
         (300, 8, 128, 64, "bf16", False), (12, 1, 200, 16, "fp32", True), (21, 2, 32, 16, "bf16", False)]


@pytest.mark.parametrize("T,H,D,page,t,pow2", CASES)
def test_write_and_read(T, H, D, page, t, pow2):
    from paper_2011_14504_amd import iseg
    P = T // page + 3
    r = rng(T + D)
    slots = r.permutation(P * page)[:T]
    xs = []
    for k in range(2):
        x = normal(10 * D + k, T, H, D) * torch.exp2(torch.from_numpy(r.integers(-6, 7, (T, H, 1)).astype(np.float64)))
        x[T // 2, 0] = 0
        # values on half-steps of a scale of 1: rounded up
        if D >= 8:
            x[0, 0] = 0
            x[0, 0, :8] = torch.tensor([7.0, 0.5, -0.5, 1.5, -1.5, 6.5, -6.5, 2.5])
        xs.append(x.to(DT[t]))
    k, v = xs
    c = iseg.kv4_cache(P, H, D, page, DEV)
    before = [x.clone() for x in c]
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    sl = torch.from_numpy(slots).to(DEV)
    # strides between tokens and heads, at odd places
    wide = torch.full((T, H + 1, D + 3), 9.0, dtype=DT[t])
    wide[:, :H, 1:D + 1] = k
    iseg.kv4_write(wide.to(DEV)[:, :H, 1:D + 1], v.to(DEV), sl.int(), c, iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX, status=st)
    assert iseg.iseg_status_read(st) == 0
    W = width(D)
    want = []
    for x, pack, b, s in ((k, key_bytes, before[0], before[1]), (v, value_bytes, before[2], before[3])):
        n, sc = _quantized(x.double(), pow2)
        full, fs = np.zeros((P * page, H, W)), np.ones((P * page, H), np.float32)
        full[slots, :, :D] = n.numpy()
        fs[slots] = sc.numpy()
        full, fs = full.reshape(P, page, H, W).swapaxes(1, 2), fs.reshape(P, page, H).swapaxes(1, 2)
        want += [pack(np.ascontiguousarray(full)), fs]
        xs.append((n.float() * sc[..., None]).to(DT[t]))
    for got, w in zip(c, want):
        assert np.array_equal(got.cpu().numpy(), w)
    for dt in DT.values():
        got = iseg.kv4_read(sl, c, D, dt, status=st)
        for g, n in zip(got, (0, 1)):
            q, s = _quantized((k, v)[n].double(), pow2)
            assert torch.equal(g.cpu(), (q.float() * s[..., None]).to(dt))
    assert iseg.iseg_status_read(st) == 0


def test_codes_are_those_of_quantize_rows():
    from paper_2011_14504_amd import iseg
    x = normal(3, 50, 4, 128).float().to(DEV)
    c = iseg.kv4_cache(4, 4, 128, 16, DEV)
    sl = torch.arange(50, device=DEV)
    for mode in (iseg.ISEG_SCALE_MAX, iseg.ISEG_SCALE_POW2):
        iseg.kv4_write(x, x, sl, c, mode)
        n, s = iseg.quantize_rows(x, bits=4, scale_mode=mode)
        want = (n.float() * s[:, None]).view(50, 4, 128)
        k, v = iseg.kv4_read(sl, c, 128)
        assert torch.equal(k, want) and torch.equal(v, want)


@pytest.mark.parametrize("t", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("pow2", [False, True])
def test_codes_beside_the_half_steps(t, pow2):
    """Elements on half-steps of their row's scale, as far as the type has them, and
    its next numbers to either side; scales from the least to the largest."""
    from paper_2011_14504_amd import iseg
    r, rows, D = rng(5), 400, 128
    info = torch.finfo(DT[t])
    lo, hi = max(-50.0, np.log2(info.tiny) + 8), min(125.0, np.log2(info.max) - 1)
    big = torch.from_numpy(np.exp2(r.uniform(lo, hi, rows))).to(DT[t])
    big[:len(big) // 2] = (big[:len(big) // 2].double() / 7).to(DT[t]) * 7          # multiples of 7, where a tie is a number of the type
    _, s = _quantized(big.double()[:, None], pow2)
    half = (torch.arange(D) % 16 - 7.5)[None] * s.double()[:, None]
    x = half.clamp(-info.max, info.max).to(DT[t])
    x = torch.where(x.double().abs() > big.double()[:, None], big[:, None].expand(-1, D), x)
    up, down = torch.nextafter(x, torch.full_like(x, info.max)), torch.nextafter(x, torch.full_like(x, -info.max))
    pick = torch.from_numpy(r.integers(0, 3, (rows, D)))
    x = torch.where(pick == 0, x, torch.where(pick == 1, up, down))
    x = torch.where(x.double().abs() > big.double()[:, None], big[:, None].expand(-1, D), x)
    x[:, 0] = big
    c, sl = iseg.kv4_cache(rows // 16, 1, D, 16, DEV), torch.arange(rows, device=DEV)
    n, s = _quantized(x.double(), pow2)
    for at in (sl, torch.arange(rows - 1, -1, -1, device=DEV)):
        iseg.kv4_write(x[:, None].to(DEV), x[:, None].to(DEV), at, c, iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX)
        assert torch.equal(c.k_scale[:, 0].reshape(-1)[at].cpu(), s) and torch.equal(c.v_scale, c.k_scale)
        for y in iseg.kv4_read(at, c, D):
            assert torch.equal(y[:, 0].cpu(), n.float() * s[:, None])


def test_extreme_rows():
    """Rows of zeros, of the smallest and largest numbers, of NaN and infinity."""
    from paper_2011_14504_amd import iseg
    D = 64
    x = torch.zeros(8, 1, D)
    x[1, 0, 3] = 2.0 ** -149
    x[2, 0] = torch.linspace(-1, 1, D) * 2.0 ** -60
    x[3, 0] = torch.linspace(-1, 1, D) * 3e38
    x[4, 0, 5] = float("nan")
    x[5, 0, 6] = -float("inf")
    x[6, 0] = torch.linspace(-1, 1, D) * 2.0 ** -56
    x[7, 0] = 1.0
    c = iseg.kv4_cache(1, 1, D, 16, DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    sl = torch.arange(8, device=DEV)
    ok = torch.tensor([0, 1, 2, 3, 6, 7], device=DEV)
    iseg.kv4_write(x[ok.cpu()].to(DEV), x[ok.cpu()].to(DEV), ok, c, status=st)
    assert iseg.iseg_status_read(st) == 0
    n, s = _quantized(x[ok.cpu()].double(), False)
    k, v = iseg.kv4_read(ok, c, D)
    assert torch.equal(k.cpu(), n.float() * s[..., None]) and torch.equal(v, k)
    iseg.kv4_write(x.to(DEV), x.to(DEV), sl, c, status=st)
    assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
    k, v = iseg.kv4_read(sl, c, D)
    for y in (k, v):
        assert torch.isnan(y[4:6]).all() and torch.isfinite(y[[0, 1, 2, 3, 6, 7]]).all()
    assert float(c.k_scale[0, 0, 0]) == 2.0 ** -60


def test_slots_that_are_none():
    """Negative slots are skipped without a word, others outside the cache with
    one; nothing else changes."""
    from paper_2011_14504_amd import iseg
    T, H, D, P, page = 6, 2, 96, 2, 16
    x = normal(1, T, H, D).to(torch.bfloat16).to(DEV)
    for dt in (torch.int32, torch.int64):
        c = iseg.kv4_cache(P, H, D, page, DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        sl = torch.tensor([-1, 5, -7, 17, -1, 31], dtype=dt, device=DEV)
        iseg.kv4_write(x, x, sl, c, status=st)
        assert iseg.iseg_status_read(st) == 0
        k, v = iseg.kv4_read(sl, c, D, torch.bfloat16, status=st)
        assert iseg.iseg_status_read(st) == 0
        for y in (k, v):
            assert (y[[0, 2, 4]] == 0).all() and (y[[1, 3, 5]] != 0).any(-1).all()
        left = [i for i in range(P * page) if i not in (5, 17, 31)]
        k, v = iseg.kv4_read(torch.tensor(left, device=DEV), c, D)
        assert (k == 0).all() and (v == 0).all()
        c0 = [t.clone() for t in c]
        out = torch.tensor([P * page, P * page + 5, 2 ** 31 - 1, -1, -1, -1], dtype=dt, device=DEV)
        iseg.kv4_write(x, x, out, c, status=st)
        assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_RANGE
        assert all(torch.equal(a, b) for a, b in zip(c, c0))
        iseg.iseg_status_clear(st)
        k, _ = iseg.kv4_read(out, c, D, status=st)
        assert (k == 0).all() and iseg.iseg_status_read(st) == iseg.ISEG_DEV_RANGE


def test_empty_calls():
    from paper_2011_14504_amd import iseg
    c = iseg.kv4_cache(2, 2, 64, 16, DEV)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    x = torch.empty(0, 2, 64, device=DEV)
    iseg.kv4_write(x, x, none, c)
    k, v = iseg.kv4_read(none, c, 64)
    assert k.shape == (0, 2, 64) and v.shape == (0, 2, 64)


def test_a_cache_past_32_bits():
    """A cache whose keys lie past 2^32 bytes: slots at both ends."""
    from paper_2011_14504_amd import iseg
    H, D, page = 8, 128, 256
    P = (1 << 32) // (H * page * 64) + 40
    c = iseg.kv4_cache(P, H, D, page, DEV)
    x = normal(4, 4, H, D).to(torch.bfloat16).to(DEV)
    y = normal(5, 4, H, D).to(torch.bfloat16).to(DEV)
    sl = torch.tensor([0, P * page - 1, P * page - 17, (P - 20) * page + 3], device=DEV)
    iseg.kv4_write(x, y, sl, c)
    small = iseg.kv4_cache(1, H, D, 16, DEV)
    at = torch.arange(4, device=DEV)
    iseg.kv4_write(x, y, at, small)
    for a, b in zip(iseg.kv4_read(sl, c, D), iseg.kv4_read(at, small, D)):
        assert torch.equal(a, b) and (a != 0).any()
