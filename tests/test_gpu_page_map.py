"""Pages, slots and positions of a step against a loop over the requests."""
import numpy as np
import pytest
import torch

from lm_util import DEV
from serve_util import rng

pytestmark = pytest.mark.gpu


def _loop(ctx, new, table, held, free, n_free, page, n_pages, T):
    """The step's results, and whether something did not fit."""
    table, held, bad = table.copy(), held.copy(), False
    B, cols = table.shape
    left = n_free
    if not 0 <= left <= len(free):
        bad, left = True, min(max(left, 0), len(free))
    start, pos, slots, kv_len = [0], [], [], []
    for b in range(B):
        c, n = max(int(ctx[b]), 0), max(int(new[b]), 0)
        bad |= ctx[b] < 0 or new[b] < 0 or not 0 <= held[b] <= cols
        h = min(max(int(held[b]), 0), cols)
        want = -(-(c + n) // page)
        if want > cols:
            bad, want = True, cols
        got = h
        for col in range(h, want):
            if left > 0:
                left -= 1
                got += 1
                pg = free[left]
                table[b, col] = pg if 0 <= pg < n_pages else -1
                bad |= not 0 <= pg < n_pages
            else:
                bad = True
                table[b, col] = -1
        for i in range(n):
            p = c + i
            col = p // page
            pg = table[b, col] if col < cols else -1
            ok = 0 <= pg < n_pages
            bad |= not ok
            pos.append(p)
            slots.append(pg * page + p % page if ok else -1)
        start.append(start[-1] + n)
        kv_len.append(c + n)
        held[b] = got
    bad |= len(pos) > T
    pos, slots = (pos + [0] * T)[:T], (slots + [-1] * T)[:T]
    return dict(table=table, q_start=start, kv_len=kv_len, positions=pos, slots=slots, held=held, n_free=[left]), bad


def _compare(ctx, new, table, held, free, n_free, page, n_pages, T, in_place=False, strided=False):
    from paper_2011_14504_amd import iseg
    want, bad = _loop(ctx, new, table, held, free, n_free, page, n_pages, T)
    g = lambda v: torch.from_numpy(np.asarray(v, dtype=np.int32)).to(DEV)  # noqa: E731
    tab = g(table)
    if strided:
        buf = torch.full((table.shape[0], table.shape[1] + 3), -9, dtype=torch.int32, device=DEV)
        buf[:, 1:-2] = tab
        tab = buf[:, 1:-2]
    hg, fg = g(held), g([n_free])
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = iseg.page_map(g(ctx), g(new), tab, hg, g(free), fg, page=page, n_pages=n_pages, n_tokens=T, in_place=in_place, status=st)
    assert iseg.iseg_status_read(st) == (iseg.ISEG_DEV_RANGE if bad else 0)
    for name, got in zip(("table", "q_start", "kv_len", "positions", "slots", "held", "n_free"), (tab,) + out):
        w = np.asarray(want[name]).astype(np.int32)
        assert np.array_equal(got.cpu().numpy(), w), (name, np.argwhere(got.cpu().numpy() != w)[:5])
    if in_place:
        assert out[4] is hg and out[5] is fg
    if strided:
        assert (buf[:, 0] == -9).all() and (buf[:, -2:] == -9).all()


def _state(seed, B, ctx_max, new_max, page, spare=3, idle=0.0):
    r = rng(seed)
    ctx = r.integers(0, ctx_max + 1, B)
    new = r.integers(0, new_max + 1, B)
    new[r.random(B) < idle] = 0
    held = -(-ctx // page) + (r.random(B) < 0.2)
    need = int(np.maximum(-(-(ctx + new) // page) - held, 0).sum())
    cols = int(max((-(-(ctx + new) // page)).max(initial=0), held.max(initial=0))) + 2
    P = int(held.sum()) + need + spare
    perm = r.permutation(P)
    table = np.full((B, cols), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.concatenate((perm[at:], r.integers(0, P, 5)))
    return dict(ctx=ctx, new=new, table=table, held=held, free=free, n_free=P - at, page=page, n_pages=P, T=int(new.sum()))


@pytest.mark.parametrize("B,ctx,new,page", [(1, 0, 1, 16), (1, 100, 1, 16), (1, 0, 5000, 16), (3, 50, 40, 1), (7, 200, 9, 48), (64, 3000, 1, 16),
                                            (257, 900, 5, 64), (1025, 300, 3, 16), (2100, 100, 20, 32), (5000, 40, 2, 16), (40, 10, 1000, 128)])
def test_against_the_loop(B, ctx, new, page):
    for k in range(2):
        _compare(**_state(B + k, B, ctx, new, page, idle=0.3 * k), in_place=bool(k), strided=bool(k))


def test_rows_behind_the_last_request():
    s = _state(4, 9, 100, 12, 16)
    s["T"] += 37
    _compare(**s)
    s = _state(4, 9, 100, 0, 16)
    s["T"] = 20
    _compare(**s)


def test_too_few_pages():
    """Requests in order take what there is; tokens without a page get no slot."""
    s = _state(5, 30, 100, 40, 16, spare=0)
    for short in (1, 3, s["n_free"]):
        t = dict(s, n_free=s["n_free"] - short)
        _compare(**t)


def test_too_few_columns_and_tokens():
    s = _state(6, 12, 100, 60, 16)
    t = dict(s, table=np.ascontiguousarray(s["table"][:, :s["held"].max()]))
    _compare(**t)
    _compare(**dict(s, T=s["T"] - 5))
    _compare(**dict(s, T=0))


def test_bad_state():
    s = _state(7, 12, 100, 30, 16)
    for name, at, v in (("ctx", 3, -5), ("new", 2, -1), ("held", 4, -2), ("held", 4, 1000)):
        t = dict(s, **{name: s[name].copy()})
        t[name][at] = v
        t["T"] = int(np.maximum(t["new"], 0).sum())
        _compare(**t)
    t = dict(s, table=s["table"].copy(), free=s["free"].copy())
    t["table"][5, :2] = [s["n_pages"], -4]
    t["free"][s["n_free"] - 2] = s["n_pages"] + 7
    t["ctx"] = s["ctx"].copy()
    t["ctx"][5] = 0
    _compare(**t)
    _compare(**dict(s, n_free=-3))
    _compare(**dict(s, n_free=len(s["free"]) + 1))


def test_nothing():
    from paper_2011_14504_amd import iseg
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    out = iseg.page_map(none, none, torch.empty(0, 4, dtype=torch.int32, device=DEV), none, none, torch.zeros(1, dtype=torch.int32, device=DEV),
                        page=16, n_pages=0, n_tokens=3)
    assert out[0].tolist() == [0] and out[2].tolist() == [0, 0, 0] and out[3].tolist() == [-1, -1, -1] and out[5].tolist() == [0]
