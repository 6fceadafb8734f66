"""Plain 64-bit references of the hybrid calls (paged append, tree attention, sampling), on the CPU, and their inputs."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2608_20961_amd import workload as wl

BF, F32 = torch.bfloat16, torch.float32


def angles(positions, rot, base=1e4):
    if rot == 0:
        return None, None
    a = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return a.cos().float(), a.sin().float()


def rotate64(x, pos, cos, sin):
    """x [..., N, d] at positions pos [N]."""
    x = x.double()
    if cos is None:
        return x
    h = cos.shape[1]
    c, s = cos[pos].double(), sin[pos].double()
    a, b = x[..., :h], x[..., h:2 * h]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * h:]], -1)


def ancestors(parent):
    """bool [N, N]: which nodes each one sees (its ancestors and itself); a bad parent counts as -1."""
    N = len(parent)
    sees = np.zeros((N, N), dtype=bool)
    for t in range(N):
        if 0 <= parent[t] < t:
            sees[t] = sees[parent[t]]
        sees[t, t] = True
    return torch.from_numpy(sees)


class Context:
    """A paged cache of given lengths, its pages shuffled, everything that no call may use NaN, and -1 past the pages."""

    def __init__(self, seed, lens, H, d, page, dtype, more=0, shared=0, spare=3):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens, self.page, B = list(lens), page, len(lens)
        need = [-(-(n + more) // page) for n in lens]
        width = max(1, max(need) + 1)
        pool = list(rng.permutation(sum(need) + spare))
        self.n_pages = len(pool)
        self.table = torch.full((B, width), -1, dtype=torch.int32)
        self.k, self.v = (torch.full((self.n_pages, H, page, d), math.nan, dtype=dtype) for _ in range(2))
        self.K, self.V = [], []
        first = max(range(B), key=lambda b: lens[b])
        order = [first] + [b for b in range(B) if b != first]
        for b in order:
            n = lens[b]
            K, V = (torch.randn(H, n, d, generator=g).to(dtype) for _ in range(2))
            common = min(shared, n)
            if b != first and common:
                K[:, :common], V[:, :common] = self.K[0][1][:, :common], self.V[0][1][:, :common]
            whole = common // page if b != first else 0
            for i in range(need[b]):
                self.table[b, i] = self.table[first, i] if i < whole else int(pool.pop())
            self.K.append((b, K)); self.V.append((b, V))
            for dst, src in ((self.k, K), (self.v, V)):
                for i in range(whole, -(-n // page)):
                    m = min(page, n - i * page)
                    dst[int(self.table[b, i]), :, :m] = src[:, i * page:i * page + m]
        self.K = [K for _, K in sorted(self.K, key=lambda x: x[0])]
        self.V = [V for _, V in sorted(self.V, key=lambda x: x[0])]

    def gpu(self):
        return (self.k.cuda(), self.v.cuda(), self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda())


def attention64(q, k, v, parents, ctx, cos, sin, scale=None):
    """o [B, Hq, N, d] in 64 bits."""
    B, Hq, N, d = q.shape
    H = k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out = torch.empty(B, Hq, N, d, dtype=torch.float64)
    for b in range(B):
        n = ctx.lens[b]
        sees = torch.ones(N, N, dtype=torch.bool).tril() if parents is None else ancestors(parents[b])
        pos = n + sees.sum(-1) - 1
        qr, kr = rotate64(q[b], pos, cos, sin), rotate64(k[b], pos, cos, sin)
        for h in range(Hq):
            hk = h // (Hq // H)
            K, V = torch.cat([ctx.K[b][hk].double(), kr[hk]]), torch.cat([ctx.V[b][hk].double(), v[b, hk].double()])
            for t in range(N):
                keep = torch.cat([torch.ones(n, dtype=torch.bool), sees[t]])
                out[b, h, t] = torch.softmax((K[keep] @ qr[h, t]) * scale, 0) @ V[keep]
    return out


def trees(seed, B, N, depth=None):
    rng = np.random.default_rng(seed)
    return np.stack([wl.random_tree(rng, N, min(N, depth or int(rng.integers(1, N + 1))), (N,)) for _ in range(B)])


# ---- sampling --------------------------------------------------------------------
def kept64(x, temperature, top_k, top_p, min_p):
    """The kept tokens' likelihoods (not normalised, others 0) of one row in 64 bits."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    order = np.lexsort((np.arange(len(x)), -x))
    with np.errstate(invalid="ignore"):
        w = np.exp(np.where(x == x.max(), 0.0, x - x.max()) / temperature)[order]
    if min_p is not None and min_p > 0:
        w = np.where(w >= min(min_p, 1.0) * w[0], w, 0.0)
    if top_k is not None and top_k > 0:
        w[top_k:] = 0.0
    if top_p is not None and top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        w = np.where((before < max(top_p, 0.0) * w.sum()) | (np.arange(len(w)) == 0), w, 0.0)
    out = np.zeros(len(x))
    out[order] = w
    return out
