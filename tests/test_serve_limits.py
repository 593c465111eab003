"""The serving operators at the limits that the header states, on both sides."""
import ctypes as C

import pytest
import torch

from lm_util import DEV

ONE = C.c_void_p(1 << 20)


@pytest.fixture(scope="module")
def iseg():
    from paper_2011_14504_amd import iseg
    iseg.lib()
    return iseg


@pytest.mark.parametrize("page", [16, 48, 8192])
def test_pages_up_to_2_31_slots(iseg, page):
    """n_pages page of 2^31 is accepted, by the helpers and by the entries; one page
    more is refused."""
    L, most = iseg.lib(), (1 << 31) // page

    def codes(n):
        m, k, a = iseg.PageMapGeom(2, 4, 8, 8, 10, n, page, 0), iseg.Kv4Geom(0, 1, 32, 32, 32, 32, 32, n, page, iseg.ISEG_BF16, iseg.ISEG_I32, 0), \
            iseg.Kv4AttentionGeom(0, 1, 1, 1, 32, 32, 32, 32, 32, n, 4, 4, 0, 0, 0, page, iseg.ISEG_BF16, 1, 1.0)
        return (L.iseg_page_map_ws(C.byref(m)) > 0, L.iseg_kv4_write(ONE, ONE, ONE, C.byref(k), ONE, ONE, ONE, ONE, None, None),
                L.iseg_kv4_read(ONE, ONE, ONE, ONE, ONE, C.byref(k), ONE, ONE, None, None), L.iseg_kv4_attention_ws(C.byref(a)) > 0)

    no = iseg.ISEG_ERR_UNSUPPORTED
    assert codes(most) == (True, iseg.ISEG_OK, iseg.ISEG_OK, True)
    assert codes(most + 1) == (False, no, no, False)
    assert iseg.kv4_cache(most, 1, 32, page, "meta").k.shape[0] == most
    with pytest.raises(ValueError, match="32 bits"):
        iseg.kv4_cache(most + 1, 1, 32, page, "meta")


def test_tokens_and_heads_of_a_call(iseg):
    """ceil(T / 16) H of 2^25 - 1 and more is refused before any work."""
    L = iseg.lib()
    for T, H in ((8177, 1 << 16), (8192, 1 << 16), (1 << 28, 2), ((1 << 31) - 1, 1), (16 * ((1 << 25) - 2) + 1, 1)):
        g = iseg.Kv4Geom(T, H, 8, H * 8, 8, H * 8, 8, 4, 16, iseg.ISEG_BF16, iseg.ISEG_I32, 0)
        assert L.iseg_kv4_write(ONE, ONE, ONE, C.byref(g), ONE, ONE, ONE, ONE, None, None) == iseg.ISEG_ERR_UNSUPPORTED, (T, H)
        assert L.iseg_kv4_read(ONE, ONE, ONE, ONE, ONE, C.byref(g), ONE, ONE, None, None) == iseg.ISEG_ERR_UNSUPPORTED, (T, H)


@pytest.mark.gpu
def test_the_last_slots_of_2_31(iseg):
    """A step that takes the last of 2^27 pages of 16 tokens."""
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    table = torch.full((1, 2), -1, dtype=torch.int32, device=DEV)
    out = iseg.page_map(i32(0), i32(17), table, i32(0), i32(0, (1 << 27) - 1), i32(2), page=16, n_pages=1 << 27, n_tokens=18, status=st)
    assert iseg.iseg_status_read(st) == 0 and table.tolist() == [[(1 << 27) - 1, 0]]
    assert out[3].tolist() == list(range((1 << 31) - 16, 1 << 31)) + [0, -1]


@pytest.mark.gpu
def test_more_than_2_27_rows(iseg):
    """2100 tokens of 2^16 heads, most of them in no slot: the others' bytes are those
    of a call of their own."""
    T, H, D = 2100, 1 << 16, 8
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    x, y = (torch.randn(T, 1, D, device=DEV, generator=torch.Generator(DEV).manual_seed(s)).half().expand(T, H, D) for s in (1, 2))
    where = {0: 3, 17: 15, 1046: 0, 2047: 7, 2048: 8, T - 1: 12}
    slots = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    for t, s in where.items():
        slots[t] = s
    big, own = (iseg.kv4_cache(1, H, D, 16, DEV) for _ in range(2))
    iseg.kv4_write(x, y, slots, big, status=st)
    at = torch.tensor(list(where), device=DEV)
    for t in where:
        iseg.kv4_write(x[t:t + 1, :4096], y[t:t + 1, :4096], slots[t:t + 1], iseg.Kv4Cache(*(c[:, :4096] for c in own)), status=st)
    for a, b in zip(big, own):
        assert torch.equal(a[:, :4096], b[:, :4096])
        assert torch.equal(a, a[:, :1].expand_as(a))          # every head is the same
    k, v = iseg.kv4_read(slots, big, D, torch.float16, status=st)
    few, _ = iseg.kv4_read(slots[at], big, D, torch.float16, status=st)
    assert torch.equal(k[at], few) and torch.equal(v[:, :1].expand_as(v), v)
    none = torch.ones(T, dtype=torch.bool, device=DEV)
    none[at] = False
    assert (k[none] == 0).all() and (v[none] == 0).all() and iseg.iseg_status_read(st) == 0
