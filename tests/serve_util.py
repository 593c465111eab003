"""Shared parts of the tests of the serving operators: the 4-bit cache in its
layout, built here by loops and permutations of its own, and the formulas in 64
bits."""
import math

import numpy as np
import torch

from lm_util import DEV, DT


def rng(seed):
    return np.random.default_rng(seed)


def width(D):
    return -(-D // 32) * 32 if D <= 128 else -(-D // 64) * 64


def key_bytes(n):
    """Codes [..., W] (numpy, -7 .. 7) in the layout of a key row."""
    u = (n.astype(np.int64) + 8).reshape(*n.shape[:-1], -1, 8)
    word = np.zeros(u.shape[:-1], dtype=np.uint64)
    for e in range(8):
        word |= u[..., e].astype(np.uint64) << np.uint64((e & 1) * 16 + (e >> 1) * 4)
    return word.astype("<u4").view(np.uint8).reshape(*n.shape[:-1], -1)


def value_bytes(n):
    """Codes [P, H, page, W] in the tiles of the values."""
    P, H, page, W = n.shape
    out = np.zeros((P, H, page // 16, 8 * W), dtype=np.uint8)
    u = (n.astype(np.int64) + 8).astype(np.uint8)
    for t in range(16):
        g, j = divmod(t, 4)
        for i in range(W // 32):
            for c in range(16):
                at = ((4 * c + g) * (W // 32) + i) * 4 + j
                out[..., at] = u[:, :, t::16, 32 * i + c] | u[:, :, t::16, 32 * i + 16 + c] << 4
    return out


class Cache:
    """A cache of random codes and scales, on the GPU in its layout and here as
    numbers."""

    def __init__(self, seed, P, H, D, page, k_size=0.4, v_size=0.4, spread=0.0):
        r = rng(seed)
        W = width(D)
        self.D, self.page = D, page
        self.kn, self.vn = (np.clip(np.rint(r.standard_normal((P, H, page, W)) * 2.6), -7, 7) for _ in range(2))
        self.kn[..., D:] = 0
        self.vn[..., D:] = 0
        self.ks = (k_size * (0.5 + r.random((P, H, page)))).astype(np.float32)
        self.vs = (v_size * (0.2 + r.random((P, H, page))) * np.exp2(spread * (r.random((P, H, page)) - 0.5))).astype(np.float32)

    def gpu(self):
        from paper_2011_14504_amd import iseg
        return iseg.Kv4Cache(*(torch.from_numpy(x).to(DEV) for x in (key_bytes(self.kn), self.ks, value_bytes(self.vn), self.vs)))

    def rows(self, pages, n, h):
        """(keys, values) float64 [n, D] of head h over the tokens of `pages`."""
        def of(c, s):
            c = c[pages][:, h, :, :self.D].reshape(-1, self.D)[:n].astype(np.float64)
            return c * s[pages][:, h].reshape(-1)[:n].astype(np.float64)[:, None]
        return of(self.kn, self.ks), of(self.vn, self.vs)


def attention(q, cache, table, q_start, kv_len, H, scale, causal, window, page_ok=None):
    """(out, lse, size): size bounds what roundings are relative to, sum_j p_j |v_j|;
    the fourth result is scale sum_d |q_d| |k_d| at its largest over the row's keys, the
    fifth scale max_d |q_d| sum_d |k_d|."""
    T, Hq, D = q.shape
    out, size = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, reach, far = np.full((T, Hq), -math.inf), np.zeros((T, Hq)), np.zeros((T, Hq))
    G = Hq // H
    for b, kv in enumerate(kv_len):
        n = q_start[b + 1] - q_start[b]
        pages = np.asarray(table[b])[:-(-kv // cache.page)] if kv else np.zeros(0, np.int64)
        good = (pages >= 0) & (pages < len(cache.ks))
        held = np.repeat(good, cache.page)[:kv]
        for hk in range(H):
            if not kv or not n:
                continue
            K, V = cache.rows(np.where(good, pages, 0), kv, hk)
            for i in range(n):
                pos = kv - n + i
                j = np.arange(kv)
                see = held & ((j <= pos) if causal else True) & ((j > pos - window) if window else True)
                if not see.any():
                    continue
                for g in range(G):
                    x = q[q_start[b] + i, hk * G + g].astype(np.float64)
                    s = scale * (K[see] @ x)
                    m = s.max()
                    p = np.exp(s - m)
                    z = p.sum()
                    row = (q_start[b] + i, hk * G + g)
                    out[row] = (p / z) @ V[see]
                    size[row] = (p / z) @ np.abs(V[see])
                    lse[row] = m + math.log(z)
                    reach[row] = scale * (np.abs(K[see]) @ np.abs(x)).max()
                    far[row] = scale * np.abs(x).max() * np.abs(K[see]).sum(1).max()
    return out, lse, size, reach, far


def table_of(seed, held, P, cols):
    """Block tables of requests that hold `held` pages of P, anywhere; -1 beyond."""
    perm = rng(seed).permutation(P)
    t = np.full((len(held), cols), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(held):
        t[b, :n] = perm[at:at + n]
        at += n
    return t


def typed(x, t):
    """float64 numpy as the values of type t: (GPU tensor, float64 of what it holds)."""
    y = torch.from_numpy(np.asarray(x)).to(DT[t])
    return y.to(DEV), y.double().numpy()
