"""Rows whose sum of squares leaves float32's range on either side."""
import pytest
import torch

from lm_util import DEV, DT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("D", [64, 33])
def test_rows_out_of_range_set_the_status(t, D):
    """Squares that are no normal float32 in sum, with nothing from eps, leave a factor
    without its bits: told as the rows beyond the range are.  Rows beside them, and the
    same ones with an eps, are what they are without them."""
    from paper_2011_14504_amd import iseg
    gen = torch.Generator().manual_seed(D)
    x = torch.randn(5, 2, D, generator=gen).to(DT[t]).to(DEV)
    pos, freq = torch.arange(5, device=DEV), iseg.rope_frequencies(16, device=DEV)
    for e, eps, said in ((-70, 0.0, True), (-80, 0.0, True), (None, 0.0, True), (-55, 0.0, False), (-70, 1e-6, False), (None, 1e-6, False), (70, 0.0, True), (70, 1e-6, True),
                         (55, 0.0, False)):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        want, _ = iseg.qk_norm_rope_fwd(x, None, pos, freq, eps=eps, status=st)
        assert iseg.iseg_status_read(st) == 0
        y = x.clone()
        y[3, 1] = 0 if e is None else y[3, 1] * 2.0 ** e
        got, _ = iseg.qk_norm_rope_fwd(y, None, pos, freq, eps=eps, status=st)
        assert iseg.iseg_status_read(st) == (iseg.ISEG_DEV_NONFINITE if said else 0), (e, eps)
        keep = torch.ones(5, 2, dtype=torch.bool, device=DEV)
        keep[3, 1] = False
        assert torch.equal(got[keep], want[keep])
        if not said and eps == 0.0:
            assert torch.equal(got, want)        # a power of two changes no bit of the quotient
        if not said and e is None:
            assert (got[3, 1] == 0).all()
