"""Writing and reading the 4-bit cache four tokens at a time, as calls of 8192 and
more token-heads do: the bytes, the scales and the values, exactly."""
import numpy as np
import pytest
import torch

from lm_util import DEV, DT, normal
from serve_util import key_bytes, rng, value_bytes, width

pytestmark = pytest.mark.gpu


def _quantized(x, pow2):
    """Codes and float32 scales of rows of float64 x; 0 and NaN for one that is not finite."""
    big = x.abs().amax(-1)
    s = torch.ldexp(torch.ones_like(big), torch.frexp(big)[1] - 3) if pow2 else big / 7
    s = torch.where(big > 0, s, torch.zeros_like(s)).float().clamp_min(2.0 ** -60)
    n = torch.floor(x / s.double()[..., None] + 0.5).clamp(-7, 7)
    odd = ~torch.isfinite(x).all(-1)
    s[odd] = float("nan")
    n[odd] = 0
    return n, s


def _slots(kind, r, T, P, page, off, wide):
    """Slots of T tokens: runs of pages from place `off` on, that with tokens without a
    slot and with slots past the cache among them, any order, runs backwards."""
    if kind == "any":
        return r.permutation(P * page)[:T].astype(np.int64)
    at = np.arange(T) + off
    s = r.permutation(P)[at // page] * page + at % page
    if kind == "back":
        s = s[::-1].copy()
    if kind == "holes":
        lost = r.random(T)
        s[lost < 0.1] = -1 if not wide else -(1 << 40)
        s[(lost >= 0.1) & (lost < 0.15)] = P * page
        s[(lost >= 0.15) & (lost < 0.2)] = (1 << 31) - 1 if not wide else (1 << 40) + 5
    return s


CASES = [(1024, 8, 128, 16, "bf16", False, "runs", 0), (1025, 8, 128, 64, "bf16", True, "runs", 1), (1027, 8, 64, 32, "fp16", False, "runs", 2),
         (1029, 8, 80, 16, "bf16", False, "runs", 3), (1039, 8, 96, 48, "fp32", True, "runs", 4), (1041, 8, 192, 16, "bf16", False, "runs", 6),
         (1200, 7, 256, 64, "fp32", False, "runs", 5), (1031, 9, 36, 16, "fp16", True, "holes", 0), (8203, 1, 7, 16, "fp32", False, "holes", 3),
         (1300, 7, 128, 16, "bf16", False, "holes", 2), (1111, 8, 192, 32, "fp16", False, "holes", 1), (1050, 8, 80, 16, "fp32", True, "any", 0),
         (1037, 8, 128, 128, "fp16", False, "any", 0), (4100, 2, 32, 16, "bf16", True, "any", 0), (1055, 8, 256, 16, "bf16", False, "back", 0),
         (2049, 5, 96, 16, "bf16", False, "back", 3), (30, 300, 64, 16, "bf16", False, "runs", 1), (17, 500, 24, 16, "fp32", False, "holes", 0)]


@pytest.mark.parametrize("T,H,D,page,t,pow2,kind,off", CASES)
def test_write_and_read(T, H, D, page, t, pow2, kind, off):
    from paper_2011_14504_amd import iseg
    assert T * H >= 8192
    r, P = rng(T + D), (T + off) // page + 3
    wide = T % 2 == 1
    slots = _slots(kind, r, T, P, page, off, wide)
    held = (slots >= 0) & (slots < P * page)
    xs = []
    for k in range(2):
        x = normal(10 * D + k, T, H, D) * torch.exp2(torch.from_numpy(r.integers(-6, 7, (T, H, 1)).astype(np.float64)))
        x[T // 2, 0] = 0
        # on half-steps of a scale of 1, in every token of a group
        x[4:9, 0] = 0
        x[4:9, 0, :7] = torch.tensor([7.0, 0.5, -0.5, 1.5, -1.5, 6.5, -6.5])
        x[13 + k, H - 1, D - 1] = float("nan")
        x[15 - k, 0, 0] = -float("inf")
        xs.append(x.to(DT[t]))
    k, v = xs
    c = iseg.kv4_cache(P, H, D, page, DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    sl = torch.from_numpy(slots).to(DEV) if wide else torch.from_numpy(slots.astype(np.int32)).to(DEV)
    # strides between tokens and heads, at odd places
    buf = torch.full((T, H + 1, D + 3), float("nan"), dtype=DT[t])
    buf[:, :H, 1:D + 1] = k
    iseg.kv4_write(buf.to(DEV)[:, :H, 1:D + 1], v.to(DEV), sl, c, iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX, status=st)
    said = (0 if held.all() or (slots < P * page).all() else iseg.ISEG_DEV_RANGE) | (iseg.ISEG_DEV_NONFINITE if held[13:16].any() else 0)
    assert iseg.iseg_status_read(st) == said
    W = width(D)
    values = []
    for i, (x, pack) in enumerate(((k, key_bytes), (v, value_bytes))):
        n, sc = _quantized(x.double(), pow2)
        full, fs = np.zeros((P * page, H, W)), np.ones((P * page, H), np.float32)
        full[slots[held], :, :D] = n.numpy()[held]
        fs[slots[held]] = sc.numpy()[held]
        full, fs = full.reshape(P, page, H, W).swapaxes(1, 2), fs.reshape(P, page, H).swapaxes(1, 2)
        assert np.array_equal(c[2 * i].cpu().numpy(), pack(np.ascontiguousarray(full)))
        assert np.array_equal(c[2 * i + 1].cpu().numpy(), fs, equal_nan=True)
        y = n.float() * sc[..., None]
        y[torch.from_numpy(~held)] = 0
        values.append(y)
    for dt in DT.values():
        st.zero_()
        for g, y in zip(iseg.kv4_read(sl, c, D, dt, status=st), values):
            assert torch.equal(torch.nan_to_num(g.cpu(), 9.0), torch.nan_to_num(y.to(dt), 9.0))
        assert iseg.iseg_status_read(st) == (said & iseg.ISEG_DEV_RANGE)


@pytest.mark.parametrize("t", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("pow2", [False, True])
def test_codes_beside_the_half_steps(t, pow2):
    """Elements on half-steps of their row's scale, as far as the type has them, and
    its next numbers to either side; scales from the least to the largest."""
    from paper_2011_14504_amd import iseg
    r, rows, D = rng(5), 8208, 64
    info = torch.finfo(DT[t])
    lo, hi = max(-50.0, np.log2(info.tiny) + 8), min(125.0, np.log2(info.max) - 1)
    big = torch.from_numpy(np.exp2(r.uniform(lo, hi, rows))).to(DT[t])
    big[:rows // 2] = (big[:rows // 2].double() / 7).to(DT[t]) * 7          # multiples of 7, where a tie is a number of the type
    _, s = _quantized(big.double()[:, None], pow2)
    half = (torch.arange(D) % 16 - 7.5)[None] * s.double()[:, None]
    x = half.clamp(-info.max, info.max).to(DT[t])
    x = torch.where(x.double().abs() > big.double()[:, None], big[:, None].expand(-1, D), x)
    up, down = torch.nextafter(x, torch.full_like(x, info.max)), torch.nextafter(x, torch.full_like(x, -info.max))
    pick = torch.from_numpy(r.integers(0, 3, (rows, D)))
    x = torch.where(pick == 0, x, torch.where(pick == 1, up, down))
    x = torch.where(x.double().abs() > big.double()[:, None], big[:, None].expand(-1, D), x)
    x[:, 0] = big
    c = iseg.kv4_cache(rows // 16, 1, D, 16, DEV)
    n, s = _quantized(x.double(), pow2)
    order = torch.arange(rows, device=DEV)
    for at in (order, order.flip(0), order.roll(1)):
        iseg.kv4_write(x[:, None].to(DEV), x[:, None].to(DEV), at, c, iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX)
        assert torch.equal(c.k_scale[:, 0].reshape(-1)[at].cpu(), s) and torch.equal(c.v_scale, c.k_scale)
        for y in iseg.kv4_read(at, c, D):
            assert torch.equal(y[:, 0].cpu(), n.float() * s[:, None])
