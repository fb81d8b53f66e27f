"""Definitions of the paged key-value cache's operators in 64 bits, slot by slot, and a pool to run them on."""
import math

import torch

from gpu_util import DEV

NAN16 = 0x7FC0


class Pool:
    """Pools of random rows for sequences of `lens` slots, pages in random order; what no sequence uses holds NaN."""

    def __init__(self, lens, heads, dtype, page, max_pages=None, seed=0, room=0, layout="slots", spare=2):
        hq, hkv, dh = heads
        g = torch.Generator().manual_seed(1000 + seed)
        self.lens_list, self.heads, self.page, self.dtype = list(lens), heads, page, dtype
        self.batch = len(lens)
        self.max_pages = max_pages or max(1, -(-(max(lens) + room) // page))
        self.cap = self.max_pages * page
        n_pages = self.batch * self.max_pages + spare
        self.table = torch.randperm(n_pages, generator=g)[: self.batch * self.max_pages].view(self.batch, self.max_pages).to(torch.int32)
        rows = torch.full((2, n_pages, page, hkv, dh), float("nan"))
        used = torch.randn(2, n_pages, page, hkv, dh, generator=g)
        for b, n in enumerate(lens):
            for p in range(-(-n // page)):
                r = min(page, n - p * page)
                rows[:, self.table[b, p], :r] = used[:, self.table[b, p], :r]
        rows = rows.to(dtype).to(DEV)
        if layout == "heads":                    # [page][head][row][i]
            rows = rows.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
        elif layout == "mixed":                  # K and V of a row side by side
            rows = rows.permute(1, 2, 0, 3, 4).contiguous().permute(2, 0, 1, 3, 4)
        self.k, self.v = rows[0], rows[1]
        self.table = self.table.to(DEV)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)

    def rows(self, which, b, n=None):
        """The first n slots of sequence b in 64 bits: [n, hkv, dh]."""
        n = self.lens_list[b] if n is None else n
        pool = self.k if which == "k" else self.v
        return pool[self.table[b].long()].reshape(self.cap, *pool.shape[2:])[:n].double()


def attention(pool, q, rows, weights_in=None, scale=None, lens=None):
    """q: [n_rows, hq * dh]; rows of each sequence.  Outputs in 64 bits: out, lse, weights, and for the tolerances the largest
    sum |q||k| and the largest score."""
    hq, hkv, dh = pool.heads
    g = hq // hkv
    scale = dh ** -0.5 if scale is None else scale
    n_rows = sum(rows)
    out = torch.zeros(n_rows, hq, dh, dtype=torch.float64, device=DEV)
    lse = torch.full((n_rows, hq), -math.inf, dtype=torch.float64, device=DEV)
    weights = None if weights_in is None else weights_in.double().clone()
    q = q.double().view(-1, hq, dh)
    size, at = 0.0, 0
    for b, r in enumerate(rows):
        n = (lens or pool.lens_list)[b]
        if r and n:
            k, v = pool.rows("k", b, n), pool.rows("v", b, n)
            for h in range(hq):
                s = scale * (q[at:at + r, h] @ k[:, h // g].T)
                z = torch.logsumexp(s, 1)
                p = torch.exp(s - z[:, None])
                out[at:at + r, h] = p @ v[:, h // g]
                lse[at:at + r, h] = z
                if weights is not None:
                    weights[b, h // g, :n] += p.sum(0)
                size = max(size, float((scale * (q[at:at + r, h].abs() @ k[:, h // g].abs().T)).max()), float(s.abs().max()))
        at += r
    return out.view(n_rows, hq * dh), lse, weights, size


def relative_error(size, n, dh):
    """Bound of a softmax weight's relative error in fp32.  The score: dh products and their sum, each step off by at most 2^-23 (the tensor
    pipe truncates) of the sum of magnitudes `size`; its product with log2 e and the subtraction of the maximum or of the log of the sum:
    three roundings of at most 2^-23 of the score each (|score| <= size); exp2: 2 ulp.  The sum over n weights and the factors of at
    most 64 joins: a rounding each."""
    return 2.0 ** -23 * ((dh + 3) * size + 4 + n + 2 * 64)


def evict(weights, pos, n, budget, sink, recent, seen):
    """One KV head: (slot that each of the first min(n, budget) slots holds afterwards), from the definition."""
    if n <= budget:
        return list(range(n))
    w = [float(x) for x in weights[:n]]
    p = [int(x) for x in pos[:n]]

    def order(j):
        first = p[j] < sink or p[j] >= seen - recent
        heavy = math.inf if w[j] != w[j] else -w[j]           # NaN behind everything
        return (0, 0.0, 0, p[j], j) if first else (1, heavy, int(w[j] != w[j]), p[j], j)

    kept = set(sorted(range(n), key=order)[:budget])
    movers = iter(j for j in range(budget, n) if j in kept)
    return [j if j in kept else next(movers) for j in range(budget)]
