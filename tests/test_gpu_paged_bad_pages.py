"""Evictions over a table with entries outside the pool: a pair of slots of which one has no page is not moved, and the slot that it would have gone to
keeps its own rows, weight and position."""
import pytest
import torch

import paged_util as U
from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("with_pos", [True, False])
@pytest.mark.parametrize("heads,lens,budget,bad", [
    ((8, 4, 64), [100, 90], 40, [(0, 5)]),                     # where rows come from
    ((8, 4, 128), [100, 90], 40, [(1, 1)]),                    # where they go
    ((8, 4, 64), [100, 90, 77], 40, [(0, 0), (0, 6), (2, 2)]),
    ((8, 8, 64), [70 + b % 9 for b in range(40)], 40, [(b, b % 5) for b in range(0, 40, 3)]),          # more heads than SMs
    ((2, 2, 64), [20000], 9000, [(0, 3), (0, 562), (0, 563), (0, 1000)])])                             # a cluster; the page that the budget ends in
def test_pairs_without_a_page_stay(dtype, with_pos, heads, lens, budget, bad):
    from paper_2603_05454_b200 import LSPError, PagedKVCache
    pool = U.Pool(lens, heads, dtype, 16)
    hkv, raw = heads[1], torch.int16 if dtype == BF else torch.int32
    g = torch.Generator().manual_seed(4)
    w = torch.rand(pool.batch, hkv, pool.cap, generator=g).to(DEV)
    pos = torch.stack([torch.randperm(pool.cap, generator=g) for _ in range(pool.batch * hkv)]).view(w.shape).to(torch.int32).to(DEV)
    slots = torch.arange(pool.cap, dtype=torch.int32, device=DEV)
    table = pool.table.long()
    for i, (b, p) in enumerate(bad):
        pool.table[b, p] = [-1, pool.k.shape[0], -2 ** 31, 2 ** 31 - 1][i % 4]
    good = ((pool.table >= 0) & (pool.table < pool.k.shape[0])).cpu()
    k, v = pool.k.clone(), pool.v.clone()
    w_out, p_out = torch.full_like(w, 7.0), torch.full_like(pos, -7)
    want_w, want_p, want_k, want_v = w_out.clone(), p_out.clone(), k.clone(), v.clone()
    kept_apart = 0
    for b, n in enumerate(lens):
        for h in range(hkv):
            p = pos[b, h] if with_pos else slots
            place = torch.tensor(U.evict(w[b, h].cpu(), p.cpu(), n, budget, 2, 5, pool.cap if with_pos else n), dtype=torch.long)
            to = torch.arange(len(place))
            moved = (place != to) & good[b, to // 16] & good[b, place // 16]
            kept_apart += int(((place != to) & ~moved).sum())
            place, to, moved = torch.where(moved, place, to).to(DEV), to.to(DEV), moved.to(DEV)
            want_w[b, h, :len(place)] = w[b, h, place]
            want_p[b, h, :len(place)] = p[place]
            for new, old in ((want_k, k), (want_v, v)):
                new[table[b, to[moved] // 16], to[moved] % 16, h] = old[table[b, place[moved] // 16], place[moved] % 16, h]
    assert kept_apart > 0
    lens_out = torch.zeros_like(pool.lens)
    c = PagedKVCache(pool.k, pool.v, pool.table, n_heads=heads[0])
    c.evict(w, pool.lens, budget, w_out, lens_out, n_sink=2, n_recent=5, pos=pos if with_pos else None, pos_out=p_out,
            seen=torch.full_like(pool.lens, pool.cap) if with_pos else None)
    with pytest.raises(LSPError) as e:
        c.check()
    assert "status 2)" in str(e.value)
    assert lens_out.tolist() == [min(n, budget) for n in lens]
    assert torch.equal(pool.k.view(raw), want_k.view(raw)) and torch.equal(pool.v.view(raw), want_v.view(raw))
    assert torch.equal(p_out, want_p) and torch.equal(w_out, want_w)
