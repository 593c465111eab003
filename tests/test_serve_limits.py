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


@pytest.mark.gpu
def test_the_last_slots_of_2_31(iseg):
    """A step that takes the last of 2^27 pages of 16 tokens."""
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    table = torch.full((1, 2), -1, dtype=torch.int32, device=DEV)
    out = iseg.page_map(i32(0), i32(17), table, i32(0), i32(0, (1 << 27) - 1), i32(2), page=16, n_pages=1 << 27, n_tokens=18, status=st)
    assert iseg.iseg_status_read(st) == 0 and table.tolist() == [[(1 << 27) - 1, 0]]
    assert out[3].tolist() == list(range((1 << 31) - 16, 1 << 31)) + [0, -1]
