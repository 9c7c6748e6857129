"""Sequences in pages for the tests of the paged cache: tables in a pool's order, every row that no sequence has spoilt."""
import numpy as np
import torch

D = 128


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Paged:
    """Caches of sequences with ``rows[s]`` rows each.  NaN and infinity in all other rows of the pool, entries behind a sequence's last page that
    name no page; ``width``: entries of a sequence's part of the table (default: one more than the longest needs)."""

    def __init__(self, rows, Hkv, page, *, seed=0, spare=2, width=None, pages=None, scale=1.0):
        rng = np.random.default_rng([seed, page, Hkv] + list(rows))
        g = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-r // page) for r in rows]
        self.page, self.n_pages = page, sum(need) + spare if pages is None else pages
        order = rng.permutation(self.n_pages)
        table = np.full((len(rows), max(need) + 1 if width is None else width), 2 ** 31 - 1, np.int64)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = order[at:at + n]
            at += n
        self.table_host = table
        self.table = i32(table)
        self.k = (scale * torch.randn(self.n_pages, page, Hkv, D, generator=g, device="cuda")).bfloat16()
        self.v = torch.randn(self.n_pages, page, Hkv, D, generator=g, device="cuda").bfloat16()
        live = torch.zeros(self.n_pages * page, dtype=torch.bool, device="cuda")
        for s, r in enumerate(rows):
            live[self.rows(s, 0, r)] = True
        self.k.flatten(0, 1)[~live] = float("nan")
        self.v.flatten(0, 1)[~live] = float("inf")

    def rows(self, s, first, last):
        """Rows of the caches as one array."""
        j = np.arange(first, last)
        return torch.tensor(self.table_host[s, j // self.page] * self.page + j % self.page, dtype=torch.long, device="cuda")

    def keys(self, s, n):
        return self.k.flatten(0, 1)[self.rows(s, 0, n)]

    def values(self, s, n):
        return self.v.flatten(0, 1)[self.rows(s, 0, n)]


def attention(q, K, V, ctx, scale):
    """(out, sum p |v|, lse, p) in 64 bits of tokens q [n][H][D] over K, V [ctx + n][Hkv][D]; p [Hkv][group][n][rows]."""
    n, H, _ = q.shape
    Hkv = K.shape[1]
    K, V = K.double().transpose(0, 1)[:, None], V.double().transpose(0, 1)[:, None]
    qq = q.double().view(n, Hkv, H // Hkv, D).permute(1, 2, 0, 3)
    x = scale * (qq @ K.transpose(2, 3))
    x.masked_fill_(torch.arange(ctx + n, device="cuda") > ctx + torch.arange(n, device="cuda")[:, None], -torch.inf)
    p, lse = torch.softmax(x, -1), torch.logsumexp(x, -1)

    def back(t):
        return t.permute(2, 0, 1, 3).reshape(n, H, D)

    return back(p @ V), back(p @ V.abs()), lse.permute(2, 0, 1).reshape(n, H), p
