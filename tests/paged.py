"""Shared helpers of the tests of the paged cache: a cache with scattered pages, and plain fp64 forms of its operators."""
import math

import torch

D = 128


class Cache:
    """Pools, a table and mass for requests of `lens` rows, with room for `room` more each.  Pages that no request
    owns, and rows behind the last, hold NaN: whatever touches them shows."""

    def __init__(self, lens, hkv, page, seed, heads_first=True, room=0, spare=3):
        gen = torch.Generator().manual_seed(seed)
        self.gen, self.lens, self.hkv, self.page = gen, list(lens), hkv, page
        per = [-(-(n + room) // page) for n in lens]
        pages = sum(per) + spare
        order = torch.randperm(pages, generator=gen).int()
        self.table = torch.full((len(lens), max(per + [1])), -7, dtype=torch.int32)
        at = 0
        for r, k in enumerate(per):
            self.table[r, :k] = order[at:at + k]
            at += k
        self.table = self.table.cuda()
        self.k, self.v = (self.pool(pages, heads_first) for _ in range(2))
        self.mass = torch.full((pages, hkv, page), math.nan, device="cuda")
        for r, n in enumerate(lens):
            if n:
                self.put(self.k, r, 0, self.normal(n, hkv, D))
                self.put(self.v, r, 0, self.normal(n, hkv, D))
                self.put(self.mass, r, 0, self.normal(n, hkv).exp())

    def pool(self, pages, heads_first):
        shape = (pages, self.hkv, self.page, D) if heads_first else (pages, self.page, self.hkv, D)
        t = torch.full(shape, math.nan, dtype=torch.bfloat16, device="cuda")
        return t if heads_first else t.transpose(1, 2)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen).cuda()

    def where(self, r, first, n, table=None):
        t = torch.arange(first, first + n, device="cuda")
        return (self.table if table is None else table)[r].long()[t // self.page], t % self.page

    def put(self, pool, r, first, rows):
        p, o = self.where(r, first, len(rows))
        pool[p, :, o] = rows.to(pool.dtype)

    def rows(self, pool, r, n, table=None):
        p, o = self.where(r, 0, n, table)
        return pool[p, :, o]


def norm_rotate64(x, weight, eps, positions, inv_freq, interleaved):
    """x [T, H, 128] in fp64."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    n = len(inv_freq)
    if n:
        a = positions.double()[:, None, None] * torch.tensor(inv_freq, dtype=torch.float64, device=x.device)
        first, second = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
        u, w = first * a.cos() - second * a.sin(), second * a.cos() + first * a.sin()
        x = x.clone()
        if interleaved:
            x[..., 0:2 * n:2], x[..., 1:2 * n:2] = u, w
        else:
            x[..., :n], x[..., n:2 * n] = u, w
    return x


def kept64(mass, budget, window):
    """Row numbers that stay, of one head: mass is a list of floats."""
    n = len(mass)
    b = min(budget, n)
    w = min(window, b)
    key = lambda i: (-mass[i] if mass[i] == mass[i] else math.inf, i)
    nan_last = lambda i: (mass[i] != mass[i],) + key(i)
    return sorted(sorted(range(n - w), key=nan_last)[:b - w]) + list(range(n - w, n))


def attention64(q, k, v, first, scale):
    """q [n, Hq, 128] whose token i sees rows 0 .. first + i of k, v [L, Hkv, 128]: (out, lse [Hq, n], weights [Hq, n, L]).
    Rows that a token does not see have no part in its sums, whatever they hold."""
    g = q.shape[1] // k.shape[1]
    kk, vv = (x.double().repeat_interleave(g, dim=1).transpose(0, 1) for x in (k, v))
    s = torch.matmul(q.double().transpose(0, 1), kk.transpose(1, 2)) * scale
    seen = torch.arange(k.shape[0], device=k.device)[None, :] <= first + torch.arange(q.shape[0], device=k.device)[:, None]
    s = torch.where(seen, s, -math.inf)
    lse = torch.logsumexp(s, -1)
    w = torch.where(seen, torch.exp(s - lse[..., None]), 0.0)
    if torch.isfinite(vv).all():
        out = torch.matmul(w, vv)
    else:
        out = torch.stack([torch.where(seen[i][None, :, None], w[:, i, :, None] * vv, 0.0).sum(1) for i in range(q.shape[0])], dim=1)
    return out.transpose(0, 1), lse, w
