"""Attention over long sequences of the paged cache, so checked that a lost, repeated or misplaced stretch shows (see paged_long.py)."""
import math

import pytest
import torch

import paged_long as L
import paged_util as U
from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
# pages of many runs, of one, and of sizes that are no multiple of 16
SHAPES = [([30011], (7, 1, 128), 64), ([30011], (2, 2, 128), 16), ([12345, 31, 16000, 0, 4097], (4, 2, 64), 48), ([9001, 16000], (8, 2, 64), 24),
          ([30000], (3, 1, 128), 40), ([300, 30011, 299, 1, 300, 300, 300, 300], (28, 4, 128), 64)]


def _half(pool):
    return torch.finfo(pool.dtype).eps / 2


def _cache(pool, n_rows, weights):
    from paper_2603_05454_b200 import PagedKVCache
    c = PagedKVCache(pool.k, pool.v, pool.table, n_heads=pool.heads[0], max_rows=n_rows, weights=weights)
    c.workspace[4096:].fill_(0xFF)
    return c


def _fill(pool, which, b, rows):
    """rows [n, hkv, dh] to the slots of sequence b."""
    n = pool.lens_list[b]
    j = torch.arange(n, device=DEV)
    (pool.k if which == "k" else pool.v)[pool.table[b].long()[j // pool.page], j % pool.page] = rows.to(pool.dtype).to(DEV)


def _close(got, ref, tol, what):
    bad = ~((got.double() == ref) | ((got.double() - ref).abs() <= tol))
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outside"


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("lens,heads,page", SHAPES)
def test_every_slot_counts_once(dtype, rows, lens, heads, page):
    """Queries of 0: all weights are equal."""
    hq, hkv, dh = heads
    pool = U.Pool(lens, heads, dtype, page, room=2 * page)
    for b, n in enumerate(lens):
        if n:
            _fill(pool, "v", b, torch.stack([L.counted_values(n, dh).roll(h, 0) for h in range(hkv)], 1))
    q = torch.zeros(len(lens) * rows, hq * dh, dtype=dtype, device=DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((len(q), hq), 7.0, device=DEV)
    w = torch.zeros(len(lens), hkv, pool.cap, device=DEV)
    c = _cache(pool, rows, True)
    c.attention(q, pool.lens, out, lse=lse, weights_out=w)
    c.check()
    for b, n in enumerate(lens):
        for r in range(b * rows, (b + 1) * rows):
            ref = pool.rows("v", b).mean(0) if n else torch.zeros(hkv, dh, dtype=torch.float64, device=DEV)
            _close(out[r].view(hkv, hq // hkv, dh), ref[:, None].expand(-1, hq // hkv, -1), L.counted_tolerance(ref, _half(pool))[:, None], f"row {r}")
            z = torch.full((hq,), math.log(n) if n else -math.inf, dtype=torch.float64, device=DEV)
            _close(lse[r], z, 4 * 2.0 ** -22 * z.abs().nan_to_num(0, 0, 0), f"lse of row {r}")
        if n:
            # e^(0 - lse), lse in log2 units off by 2^-22 of at most 15 and the exponential by 2 ulp; rows * group of them added up
            share = torch.full((hkv, n), rows * (hq // hkv) / n, dtype=torch.float64, device=DEV)
            _close(w[b, :, :n], share, share * (4 * 2.0 ** -22 * 15 + 2.0 ** -22 + rows * (hq // hkv) * 2.0 ** -24), f"weights of sequence {b}")
        assert bool((w[b, :, n:] == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,heads,page", SHAPES)
def test_every_slot_is_found(dtype, lens, heads, page):
    """Keys of -1 and 1, a query eight times a key: that slot has all of the weight (the others' are below 2^-126, 0 in fp32), to the last
    bit."""
    hq, hkv, dh = heads
    group = hq // hkv
    pool = U.Pool(lens, heads, dtype, page, room=2 * page)
    g = torch.Generator().manual_seed(11)
    for b, n in enumerate(lens):
        _fill(pool, "k", b, 2.0 * torch.randint(2, (n, hkv, dh), generator=g) - 1)
        if n:
            s = pool.rows("k", b)[:, 0]
            s = (s[: 64] @ s.T)                            # (a few rows of the products: how alike two keys are)
            s[torch.arange(len(s)), torch.arange(len(s))] = 0
            assert float(s.max()) < dh - 16
    rows = 16
    c = _cache(pool, rows, True)
    for turn in range(24):
        target = torch.zeros(len(lens), rows, hkv, group, dtype=torch.long)
        q = torch.zeros(len(lens), rows, hkv, group, dh, dtype=torch.float64, device=DEV)
        want = torch.zeros_like(q)
        share = torch.zeros(len(lens), hkv, pool.cap, dtype=torch.float64, device=DEV)
        for b, n in enumerate(lens):
            if n:
                # ends of sequence, pages and runs, and anywhere
                t = torch.randint(n, (rows, hkv, group), generator=g)
                t[0] = n - 1 - turn % n
                t[1] = turn % n
                t[2] = (t[2] // page * page + [0, -1][turn % 2]).clamp(0, n - 1)
                target[b] = t
                k, v = pool.rows("k", b), pool.rows("v", b)
                h = torch.arange(hkv).view(1, -1, 1).expand_as(t)
                q[b], want[b] = 8 * k[t, h], v[t, h]
                share[b].index_put_((h.reshape(-1).to(DEV), t.reshape(-1).to(DEV)), torch.ones(t.numel(), dtype=torch.float64, device=DEV), accumulate=True)
        q = q.view(len(lens) * rows, hq * dh).to(dtype)
        out, w = torch.full_like(q, 7.0), torch.zeros(len(lens), hkv, pool.cap, device=DEV)
        c.attention(q, pool.lens, out, scale=1.0, weights_out=w)
        assert torch.equal(out.double().view(want.shape), want), turn
        assert torch.equal(w.double(), share), turn
    c.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,heads,page", SHAPES)
def test_random_rows_within_the_sums_that_are_formed(dtype, lens, heads, page):
    hq, hkv, dh = heads
    pool = U.Pool(lens, heads, dtype, page, room=2 * page)
    q = (2 * torch.randn(len(lens), hq * dh, generator=torch.Generator().manual_seed(5))).to(dtype).to(DEV)
    out = torch.full_like(q, 7.0)
    c = _cache(pool, 1, False)
    c.attention(q, pool.lens, out)
    c.check()
    for b, n in enumerate(lens):
        for h in range(hq):
            got = out[b:b + 1, h * dh:(h + 1) * dh]
            if n == 0:
                assert bool((got == 0).all())
                continue
            ref, magnitude, _, size, _ = L.reference(q[b:b + 1, h * dh:(h + 1) * dh], pool.rows("k", b)[:, h * hkv // hq], pool.rows("v", b)[:, h * hkv // hq], dh ** -0.5)
            _close(got, ref, L.tolerance(ref, magnitude, size, dh, _half(pool)), f"sequence {b}, head {h}")
