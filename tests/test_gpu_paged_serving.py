"""The paged cache as a server uses it: append, attention, eviction, turn after turn, thinned again and again, each turn against the definition."""
import pytest
import torch

import paged_util as U
from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,batch,page,max_pages", [((8, 4, 64), 3, 16, 20), ((4, 2, 128), 2, 24, 400), ((8, 8, 64), 40, 16, 20)])
def test_turn_after_turn_the_recent_positions_stay(dtype, heads, batch, page, max_pages):
    from paper_2603_05454_b200 import PagedKVCache
    hq, hkv, dh = heads
    rows, budget, sink, recent = 8, 96, 4, 32
    lens = [200 - 90 * b % 170 for b in range(batch)]
    pool = U.Pool(lens, heads, dtype, page, max_pages=max_pages)
    cache = PagedKVCache(pool.k, pool.v, pool.table, n_heads=hq, max_rows=rows, weights=True)
    g = torch.Generator().manual_seed(3)
    raw = torch.int16 if dtype == BF else torch.int32
    shape = (batch, hkv, pool.cap)
    w, w2 = torch.zeros(shape, device=DEV), torch.zeros(shape, device=DEV)
    pos = torch.arange(pool.cap, dtype=torch.int32, device=DEV).expand(shape).contiguous()
    pos2 = pos.clone()
    n, n2, seen, seen2 = pool.lens.clone(), pool.lens.clone(), pool.lens.clone(), pool.lens.clone()
    table = pool.table.long()
    for turn in range(14):
        new = torch.randn(batch * rows, (hq + 2 * hkv) * dh, generator=g).to(dtype).to(DEV)
        q, out = new[:, :hq * dh], torch.empty(batch * rows, hq * dh, dtype=dtype, device=DEV)
        cache.append(new[:, hq * dh:(hq + hkv) * dh], new[:, (hq + hkv) * dh:], n, n2, weights=w, pos=pos, seen=seen, seen_out=seen2)
        cache.attention(q, n2, out, weights_in=w, weights_out=w)
        before = pool.k.clone(), pool.v.clone()
        cache.evict(w, n2, budget, w2, n, n_sink=sink, n_recent=recent, pos=pos, pos_out=pos2, seen=seen2)
        cache.check()
        want = before[0].clone(), before[1].clone()
        now, total = n2.tolist(), seen2.tolist()
        for b in range(batch):
            for h in range(hkv):
                place = torch.tensor(U.evict(w[b, h].cpu(), pos[b, h].cpu(), now[b], budget, sink, recent, total[b]), device=DEV)
                to = torch.arange(len(place), device=DEV)
                for x, old in zip(want, before):
                    x[table[b, to // page], to % page, h] = old[table[b, place // page], place % page, h]
                assert torch.equal(w2[b, h, :len(place)], w[b, h, place]) and torch.equal(pos2[b, h, :len(place)], pos[b, h, place])
                held = set(pos2[b, h, :len(place)].tolist())
                assert len(held) == min(budget, now[b]) and set(range(max(0, total[b] - recent), total[b])) <= held and set(range(sink)) <= held
        assert torch.equal(pool.k.view(raw), want[0].view(raw)) and torch.equal(pool.v.view(raw), want[1].view(raw))
        assert n.tolist() == [min(budget, x) for x in now] and total == [x + rows * (turn + 1) for x in lens]
        w, w2, pos, pos2, seen, seen2 = w2, w, pos2, pos, seen2, seen
