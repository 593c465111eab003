"""Host threads that call the helpers at once: each has a workspace of its own,
and calls of two threads on one stream give the bits of calls one after the
other."""
import threading

import pytest
import torch

from lm_util import DEV, codes, normal


def _together(work, n=2):
    """work(k) in n threads that start at once; their results in order."""
    out, err, gate = [None] * n, [], threading.Barrier(n)

    def body(k):
        try:
            gate.wait(30)
            out[k] = work(k)
            gate.wait(60)                        # every thread lives until all are done
        except BaseException as e:
            err.append(e)
            gate.abort()

    ts = [threading.Thread(target=body, args=(k,)) for k in range(n)]
    for t in ts:
        t.start()
    for t in ts:
        t.join(90)
    assert not err, err
    return out


def test_every_thread_has_a_workspace_of_its_own():
    from paper_2011_14504_amd import iseg
    mine = iseg.workspace("cpu")

    def work(k):
        ws = iseg.workspace("cpu")
        assert iseg.workspace("cpu") is ws       # the next call's is the same
        return ws, ws.get(1000)

    (a, va), (b, vb) = _together(work)
    assert a is not b and a is not mine and b is not mine and va.data_ptr() != vb.data_ptr()
    assert iseg.workspace("cpu") is mine


@pytest.mark.gpu
def test_threads_on_one_stream():
    """Calls of several kernels that hand data on through the workspace: packed
    operands, a split reduction, quantized columns, partial sums of rows and of
    a cut vocabulary, and a quantized tensor's maxima."""
    from paper_2011_14504_amd import iseg
    ins = []
    for k in range(2):
        s = 100 * k
        ins.append(dict(
            a=codes(s + 1, 60, 1003).to(DEV), b=codes(s + 2, 130, 1003).to(DEV),
            c=codes(s + 3, 40, 9008).to(DEV), d=codes(s + 4, 70, 9008).to(DEV),
            x=normal(s + 5, 300, 260).float().to(DEV), dy=normal(s + 6, 300, 200).float().to(DEV),
            w=codes(s + 7, 200, 260).to(DEV), q=codes(s + 8, 300, 260).to(DEV), sc=(normal(s + 9, 300).abs() + 0.1).float().to(DEV),
            l=normal(s + 10, 2, 131072).float().to(DEV), t=torch.tensor([5, 77], device=DEV)))

    def calls(i):
        y, mean, rstd = iseg.layernorm_fwd(i["x"])
        return (iseg.matmul_i8(i["a"], i["b"]), iseg.matmul_i8(i["c"], i["d"]),
                *iseg.linear_i8_bwd(i["dy"], i["q"], i["sc"], i["w"], want_bias=True), *iseg.quantize_cols(i["x"])[:2],
                *iseg.layernorm_bwd(y, i["x"], None, mean, rstd), *iseg.logprob_fwd(i["l"], i["t"], top_k=20),
                *iseg.quantize(i["x"], 8))

    want = [calls(i) for i in ins]
    torch.cuda.synchronize()
    got = _together(lambda k: [calls(ins[k]) for _ in range(40)])
    torch.cuda.synchronize()
    for k in range(2):
        for rep in got[k]:
            for n, (g, w) in enumerate(zip(rep, want[k])):
                assert torch.equal(g, w), (k, n)
