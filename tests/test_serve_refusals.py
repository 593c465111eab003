"""Refusals of the serving operators, on the CPU: the C entries check their
arguments before anything is enqueued, the helpers before any entry."""
import ctypes as C
import math

import pytest
import torch


@pytest.fixture(scope="module")
def iseg():
    from paper_2011_14504_amd import iseg
    iseg.lib()
    return iseg


ONE = C.c_void_p(1 << 20)
BIG = 1 << 60


def test_page_map_entry(iseg):
    L = iseg.lib()

    def call(B=2, T=4, mp=8, ld=8, F=10, n_pages=20, page=16, reserved=0, ctx=ONE, table=ONE, pos=ONE, n_free=ONE, free=ONE, q_start=ONE, ws=ONE, n=BIG):
        g = iseg.PageMapGeom(B, T, mp, ld, F, n_pages, page, reserved)
        return L.iseg_page_map(ctx, ONE, ONE, free, n_free, C.byref(g), table, q_start, ONE, pos, ONE, ONE, ONE, ws, n, None, None)

    for bad in (dict(reserved=1), dict(ctx=None), dict(table=None), dict(pos=None), dict(n_free=None), dict(free=None), dict(q_start=None)):
        assert call(**bad) == iseg.ISEG_ERR_ARG, bad
    for bad in (dict(B=-1), dict(T=-1), dict(B=(1 << 31) - 1), dict(T=1 << 31), dict(mp=-1), dict(ld=7), dict(F=-1), dict(n_pages=-1), dict(page=0)):
        assert call(**bad) == iseg.ISEG_ERR_SHAPE, bad
    for bad in (dict(n_pages=(1 << 27) + 1), dict(F=1 << 31), dict(mp=1 << 31, ld=1 << 31)):
        assert call(**bad) == iseg.ISEG_ERR_UNSUPPORTED, bad
    assert call(ws=None) == iseg.ISEG_ERR_WORKSPACE and call(n=511) == iseg.ISEG_ERR_WORKSPACE
    g = iseg.PageMapGeom(-1, 4, 8, 8, 10, 20, 16, 0)
    assert L.iseg_page_map_ws(C.byref(g)) == 0 and L.iseg_page_map_ws(None) == 0


def test_qk_norm_rope_entries(iseg):
    L = iseg.lib()

    def geom(T=4, Hq=2, Hk=1, D=8, q=(16, 8), k=(8, 8), yq=(16, 8), yk=(8, 8), dq=(16, 8), dk=(8, 8), dt=iseg.ISEG_BF16, pt=iseg.ISEG_F32, pos=iseg.ISEG_I32,
             R=8, pairs=0, norm=1, eps=1e-6, ms=1.0):
        return iseg.QkNormRopeGeom(T, Hq, Hk, D, *q, *k, *yq, *yk, *dq, *dk, dt, pt, pos, R, pairs, norm, eps, ms)

    def fwd(g, q=ONE, yq=ONE, pos=ONE, freq=ONE, k=ONE):
        return L.iseg_qk_norm_rope_fwd(q, k, pos, freq, None, None, C.byref(g), yq, ONE, None, None)

    def bwd(g, dyq=ONE, dq=ONE, q=ONE, dgq=ONE, ws=ONE, n=BIG, pos=ONE):
        return L.iseg_qk_norm_rope_bwd(dyq, ONE, q, ONE, pos, ONE, None, None, C.byref(g), dq, ONE, dgq, None, ws, n, None)

    for bad in (dict(dt=iseg.ISEG_I8), dict(pt=iseg.ISEG_I32), dict(pos=iseg.ISEG_F32), dict(pairs=2), dict(norm=-1), dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan),
                dict(ms=math.inf), dict(ms=math.nan)):
        assert fwd(geom(**bad)) == iseg.ISEG_ERR_ARG and bwd(geom(**bad)) == iseg.ISEG_ERR_ARG, bad
        assert L.iseg_qk_norm_rope_bwd_ws(C.byref(geom(**bad))) == 0
    for bad in (dict(T=-1), dict(Hq=-1), dict(Hk=-1), dict(D=0, R=0), dict(R=10), dict(R=7), dict(R=-2), dict(q=(-1, 8)), dict(k=(8, -8)), dict(T=1 << 31)):
        assert fwd(geom(**bad)) == iseg.ISEG_ERR_SHAPE and bwd(geom(**bad)) == iseg.ISEG_ERR_SHAPE, bad
    for y in ((16, 7), (8, 8), (15, 8), (7, 40), (0, 8)):         # rows of the output that overlap
        assert fwd(geom(yq=y)) == iseg.ISEG_ERR_SHAPE and bwd(geom(dq=y)) == iseg.ISEG_ERR_SHAPE, y
    assert fwd(geom(D=514, R=0, q=(1028, 514), yq=(1028, 514), k=(514, 514), yk=(514, 514))) == iseg.ISEG_ERR_UNSUPPORTED
    for bad in (dict(q=None), dict(yq=None), dict(pos=None), dict(freq=None), dict(k=None)):
        assert fwd(geom(), **bad) == iseg.ISEG_ERR_ARG, bad
    for bad in (dict(dyq=None), dict(dq=None), dict(q=None), dict(pos=None)):
        assert bwd(geom(), **bad) == iseg.ISEG_ERR_ARG, bad
    assert bwd(geom(norm=0)) == iseg.ISEG_ERR_ARG               # no gamma, no gradient of it
    assert bwd(geom(), ws=None) == iseg.ISEG_ERR_WORKSPACE
    assert bwd(geom(), n=L.iseg_qk_norm_rope_bwd_ws(C.byref(geom())) - 1) == iseg.ISEG_ERR_WORKSPACE
    assert fwd(geom(T=0), q=None, yq=None, k=None) == iseg.ISEG_OK and fwd(geom(Hq=0, Hk=0), q=None, k=None, pos=None) == iseg.ISEG_OK


def test_kv4_entries(iseg):
    L = iseg.lib()

    def geom(T=4, H=2, D=64, k=(128, 64), v=(128, 64), P=3, page=16, dt=iseg.ISEG_BF16, st=iseg.ISEG_I32, mode=0):
        return iseg.Kv4Geom(T, H, D, *k, *v, P, page, dt, st, mode)

    def write(g, k=ONE, slots=ONE, kc=ONE, vs=ONE):
        return L.iseg_kv4_write(k, ONE, slots, C.byref(g), kc, ONE, ONE, vs, None, None)

    def read(g, k=ONE, slots=ONE, kc=ONE):
        return L.iseg_kv4_read(kc, ONE, ONE, ONE, slots, C.byref(g), k, ONE, None, None)

    for f in (write, read):
        for bad in (dict(dt=iseg.ISEG_I8), dict(st=iseg.ISEG_F32)):
            assert f(geom(**bad)) == iseg.ISEG_ERR_ARG, bad
        for bad in (dict(T=-1), dict(H=-1), dict(D=0), dict(page=0), dict(page=24), dict(P=-1), dict(k=(-1, 64))):
            assert f(geom(**bad)) == iseg.ISEG_ERR_SHAPE, bad
        for bad in (dict(D=257, k=(514, 257), v=(514, 257)), dict(page=8208), dict(P=1 << 28)):
            assert f(geom(**bad)) == iseg.ISEG_ERR_UNSUPPORTED, bad
        for bad in (dict(k=None), dict(slots=None), dict(kc=None), dict(kc=C.c_void_p(ONE.value + 4))):
            assert f(geom(), **bad) == iseg.ISEG_ERR_ARG, bad
        assert f(geom(T=0), k=None, slots=None) == iseg.ISEG_OK
    assert write(geom(mode=2)) == iseg.ISEG_ERR_ARG and write(geom(), vs=None) == iseg.ISEG_ERR_ARG
    for bad in (dict(k=(64, 64)), dict(v=(128, 63)), dict(k=(0, 64))):
        assert read(geom(**bad)) == iseg.ISEG_ERR_SHAPE, bad


def test_kv4_attention_entry(iseg):
    L = iseg.lib()

    def geom(T=5, B=2, Hq=4, H=2, D=64, q=(256, 64), o=(256, 64), P=9, mp=6, ld=6, mq=0, mkv=0, win=0, page=16, dt=iseg.ISEG_BF16, causal=1, scale=0.125):
        return iseg.Kv4AttentionGeom(T, B, Hq, H, D, *q, *o, P, mp, ld, mq, mkv, win, page, dt, causal, scale)

    def call(g, q=ONE, kc=ONE, table=ONE, q_start=ONE, kv=ONE, out=ONE, ws=ONE, n=BIG):
        return L.iseg_kv4_attention(q, kc, ONE, ONE, ONE, table, q_start, kv, C.byref(g), out, None, ws, n, None, None)

    for bad in (dict(dt=iseg.ISEG_I8), dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan)):
        assert call(geom(**bad)) == iseg.ISEG_ERR_ARG and L.iseg_kv4_attention_ws(C.byref(geom(**bad))) == 0, bad
    for bad in (dict(T=-1), dict(B=-1), dict(H=0), dict(Hq=3), dict(Hq=0), dict(D=0), dict(q=(-1, 64)), dict(o=(64, 64)), dict(o=(256, 60)), dict(P=-1), dict(ld=5), dict(mq=-1),
                dict(mkv=-1), dict(win=-1), dict(page=8), dict(page=40)):
        assert call(geom(**bad)) == iseg.ISEG_ERR_SHAPE, bad
    for bad in (dict(D=60), dict(D=264, q=(2000, 264), o=(2000, 264)), dict(page=8208), dict(P=1 << 28), dict(mp=1 << 27, ld=1 << 27), dict(B=1 << 25), dict(win=1 << 41),
                dict(P=1 << 24, H=4096, Hq=4096, o=(64 * 4096, 64))):
        assert call(geom(**bad)) == iseg.ISEG_ERR_UNSUPPORTED, bad
    for bad in (dict(q=None), dict(kc=None), dict(table=None), dict(q_start=None), dict(kv=None), dict(out=None), dict(kc=C.c_void_p(ONE.value + 8))):
        assert call(geom(), **bad) == iseg.ISEG_ERR_ARG, bad
    long = geom(B=1, P=10000, mp=9000, ld=9000)
    need = L.iseg_kv4_attention_ws(C.byref(long))
    assert need > 512 and call(long, n=need - 1) == iseg.ISEG_ERR_WORKSPACE and call(long, ws=None) == iseg.ISEG_ERR_WORKSPACE
    assert call(geom(T=0), q=None, out=None) == iseg.ISEG_OK and call(geom(B=0), q=None, out=None) == iseg.ISEG_OK


def test_verify_entry(iseg):
    L = iseg.lib()

    def call(B=2, S=3, V=10, t=(40, 10), d=(30, 10), dt=iseg.ISEG_F32, tt=iseg.ISEG_I32, target=ONE, tokens=ONE, n_draft=ONE, us=ONE, out=ONE, ws=ONE, n=BIG):
        g = iseg.VerifyGeom(B, S, V, *t, *d, dt, tt)
        return L.iseg_verify_drafts(target, ONE, tokens, n_draft, ONE, us, C.byref(g), out, ONE, ws, n, None, None)

    for bad in (dict(dt=iseg.ISEG_I8), dict(tt=iseg.ISEG_F32), dict(target=None), dict(tokens=None), dict(n_draft=None), dict(us=None), dict(out=None)):
        assert call(**bad) == iseg.ISEG_ERR_ARG, bad
    for bad in (dict(B=-1), dict(S=-1), dict(V=0), dict(V=1 << 31), dict(t=(-1, 10)), dict(d=(30, -1))):
        assert call(**bad) == iseg.ISEG_ERR_SHAPE, bad
    assert call(B=(1 << 16) + 1) == iseg.ISEG_ERR_UNSUPPORTED and call(S=(1 << 20) + 1) == iseg.ISEG_ERR_UNSUPPORTED
    assert call(ws=None) == iseg.ISEG_ERR_WORKSPACE and call(n=100) == iseg.ISEG_ERR_WORKSPACE
    assert call(B=0, target=None) == iseg.ISEG_OK


def _refused(f, message):
    with pytest.raises(ValueError, match=message):
        f()


def test_helpers(iseg):
    f, i = torch.float32, torch.int32
    v = lambda n, d=i: torch.zeros(n, dtype=d)  # noqa: E731
    kw = dict(page=16, n_pages=4, n_tokens=3)
    base = dict(ctx=v(2), count=v(2), table=torch.zeros(2, 4, dtype=i), held=v(2), free_pages=v(4), n_free=v(1), **kw)
    for name, bad, say in (("table", torch.zeros(3, 4, dtype=i), "table"), ("table", torch.zeros(2, 4), "table"), ("table", torch.zeros(4, 2, dtype=i).t(), "table"),
                           ("page", 0, "sizes"), ("n_tokens", -1, "sizes"), ("n_pages", 1 << 28, "32 bits"), ("ctx", v(2), "GPU tensors")):
        _refused(lambda: iseg.page_map(**dict(base, **{name: bad})), say)

    q, k, fr = torch.zeros(3, 4, 8), torch.zeros(3, 2, 8), torch.zeros(4)
    rope = lambda **o: iseg.qk_norm_rope_fwd(**dict(dict(q=q, k=k, positions=v(3), inv_freq=fr), **o))  # noqa: E731
    for o, say in ((dict(q=None, k=None), "q or k"), (dict(q=torch.zeros(3, 8)), "tokens, heads"), (dict(q=v(3).view(3, 1, 1)), "float32"), (dict(k=k[:2]), "q's tokens"),
                   (dict(k=k.half()), "q's tokens"), (dict(inv_freq=torch.zeros(5)), "half a head"), (dict(inv_freq=fr.double()), "inv_freq"), (dict(positions=v(2)), "positions"),
                   (dict(positions=torch.zeros(3)), "positions"), (dict(gamma_q=torch.zeros(7)), "gamma_q"), (dict(gamma_q=torch.zeros(8), norm=False), "norm expected"),
                   (dict(gamma_q=torch.zeros(8), gamma_k=torch.zeros(8).half()), "gamma_k"), (dict(eps=-1.0), "eps"), (dict(mscale=math.inf), "mscale"),
                   (dict(q=torch.zeros(3, 1, 513), k=None), "1 to 512"), (dict(), "GPU tensors")):
        _refused(lambda: rope(**o), say)
    _refused(lambda: iseg.qk_norm_rope_bwd(q[:2], k, q, k, v(3), fr), "dyq")
    _refused(lambda: iseg.qk_norm_rope_bwd(q, None, q, k, v(3), fr), "dyk")
    for bad in (dict(rope_dim=7), dict(rope_dim=0), dict(rope_dim=8, base=0.0), dict(rope_dim=8, factor=-1.0), dict(rope_dim=8, stretch=(100, 4, 2))):
        with pytest.raises(ValueError):
            iseg.rope_frequencies(device="cpu", **bad)

    for bad in (dict(n_pages=-1), dict(heads=0), dict(dim=0), dict(dim=257), dict(page=8), dict(page=24), dict(page=16384)):
        _refused(lambda: iseg.kv4_cache(**dict(dict(n_pages=2, heads=2, dim=64, page=16, device="cpu"), **bad)), "kv4_cache")
    _refused(lambda: iseg.kv4_cache(1 << 28, 1, 32, 16, "meta"), "32 bits")
    c = iseg.kv4_cache(2, 2, 64, 16, "cpu")
    x = torch.zeros(3, 2, 64)
    _refused(lambda: iseg.kv4_write(x, x.half(), v(3), c), "k's shape")
    _refused(lambda: iseg.kv4_write(x, x, v(3), c, scale_mode=3), "scale_mode")
    _refused(lambda: iseg.kv4_write(x, x, v(2), c), "slots")
    _refused(lambda: iseg.kv4_write(x, x, v(3, f), c), "slots")
    _refused(lambda: iseg.kv4_write(x, x, v(3), c), "GPU tensors")
    _refused(lambda: iseg.kv4_read(v(3, f), c), "slots")
    _refused(lambda: iseg.kv4_read(v(3), c, dim=100), "rows of 64 bytes")
    _refused(lambda: iseg.kv4_read(v(3), c, dtype=i), "float32")
    _refused(lambda: iseg.kv4_read(v(3), c._replace(v=c.v[:1])), "four tensors")
    _refused(lambda: iseg.kv4_read(v(3), c._replace(k_scale=c.k_scale.transpose(0, 1).contiguous().transpose(0, 1))), "dense")

    q, table = torch.zeros(3, 4, 64), torch.zeros(2, 5, dtype=i)
    at = lambda **o: iseg.kv4_attention(**dict(dict(q=q, cache=c, table=table, q_start=v(3), kv_len=v(2)), **o))  # noqa: E731
    for o, say in ((dict(q=torch.zeros(3, 4, 60)), "multiple of 8"), (dict(q=torch.zeros(3, 4)), "tokens, heads"), (dict(q=q.to(i)), "float32"), (dict(), "GPU tensors")):
        _refused(lambda: at(**o), say)
    p = torch.zeros(2, 4, 10)
    ver = lambda **o: iseg.verify_drafts(**dict(dict(target=p, draft=p[:, :3], tokens=torch.zeros(2, 3, dtype=i), n_draft=v(2), u=torch.zeros(2, 3), u_sample=torch.zeros(2)), **o))  # noqa: E731
    for o, say in ((dict(target=p[0]), "target"), (dict(draft=p), "draft"), (dict(draft=p[:, :3].half()), "draft"), (dict(tokens=torch.zeros(2, 4, dtype=i)), "tokens"),
                   (dict(tokens=torch.zeros(2, 3)), "tokens"), (dict(u=torch.zeros(2, 2)), "tokens, u"), (dict(n_draft=v(3)), "n_draft"), (dict(u_sample=torch.zeros(3)), "u_sample"),
                   (dict(), "GPU tensors")):
        _refused(lambda: ver(**o), say)
