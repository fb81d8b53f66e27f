"""The paged cache where its kernels' variants and their limits meet: tables far wider than the sequences, many sequences with offsets and several tiles
of rows, odd pages with many pairs, more heads than SMs of long sequences, the largest tables."""
import pytest
import torch

import paged_util as U
import test_gpu_paged as T
from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
SMALL, GQA, ONE = (8, 4, 64), (28, 4, 128), (1, 1, 64)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,heads,page,max_pages,rows", [
    ([70, 0, 33], SMALL, 16, 500, [1, 1, 1]), ([1, 300], GQA, 24, 700, [3, 2]), ([5], ONE, 1, 1 << 20, [2]),
    ([130, 64], ONE, 64, 1 << 14, [1, 1]), ([40, 41], (4, 4, 64), 1 << 15, 2, [1, 0])])
def test_tables_far_wider_than_the_sequences(dtype, lens, heads, page, max_pages, rows):
    pool = _wide(lens, heads, dtype, page, max_pages)
    T._check_attention(pool, rows, True, seed=2)
    w, pos = T._weights(pool, 3, ties=False) if pool.cap < 40000 else (torch.rand(pool.batch, heads[1], pool.cap, device=DEV), None)
    if pos is not None:
        T._check_evict(pool, w, pos, 32, 2, 7, seen=pool.lens + 5)
    else:
        T._check_evict(pool, w, None, 32, 2, 7, with_pos=False)


def _wide(lens, heads, dtype, page, max_pages):
    """A pool with no more pages than are used: the rest of the table names none."""
    used = U.Pool(lens, heads, dtype, page)
    table = torch.full((len(lens), max_pages), -1, dtype=torch.int32, device=DEV)
    for b, m in enumerate(lens):
        p = -(-m // page)
        table[b, :p] = used.table[b, :p]
    used.max_pages, used.cap = max_pages, max_pages * page
    used.table = table

    def narrow(which, b, k=None):
        k = used.lens_list[b] if k is None else k
        pool = used.k if which == "k" else used.v
        return pool[table[b, :max(1, -(-k // page))].long()].reshape(-1, *pool.shape[2:])[:k].double()
    used.rows = narrow
    return used


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,page,batch", [((8, 2, 64), 16, 75), ((6, 2, 128), 24, 40), ((16, 1, 64), 5, 33)])
def test_many_sequences_with_offsets_and_several_tiles(dtype, heads, page, batch):
    """Rows from none to eleven of up to 16 heads a KV head: tiles from none to eleven, two at a time."""
    lens = [(53 * b) % 211 for b in range(batch)]
    rows = [(7 * b) % 12 for b in range(batch)]
    T._check_attention(U.Pool(lens, heads, dtype, page, room=3), rows, True, seed=9)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [1, 7, 40])
@pytest.mark.parametrize("heads,rows", [((28, 4, 128), [3, 5]), ((8, 8, 64), [19, 70]), ((64, 1, 128), [1, 2])])
def test_many_pairs_over_odd_pages(dtype, page, heads, rows):
    T._check_attention(U.Pool([333, 150], heads, dtype, page, room=2), rows, True, seed=4)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_of_a_pass(dtype):
    """A block of 256 rows, as a pass has them."""
    T._check_attention(U.Pool([700, 81], (8, 2, 64), dtype, 32), [256, 130], True, seed=6)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,heads,budget", [([4200 + b for b in range(3)], (60, 60, 64), 1000), ([5000, 100, 0, 4097], (40, 40, 64), 4096)])
def test_evict_of_more_heads_than_sms_from_long_sequences(dtype, lens, heads, budget):
    pool = U.Pool(lens, heads, dtype, 16)
    g = torch.Generator().manual_seed(8)
    w = torch.rand(pool.batch, heads[1], pool.cap, generator=g)
    w = torch.where(w < 0.3, torch.zeros(()), w).to(DEV)
    key = torch.rand(pool.batch, heads[1], pool.cap, generator=g)
    T._check_evict(pool, w, torch.argsort(key, -1).to(torch.int32).to(DEV), budget, 5, 100, seen=torch.full_like(pool.lens, pool.cap))


@pytest.mark.parametrize("lens,max_pages", [([100 + b % 9 for b in range(40)], 300), ([100 + b % 9 for b in range(40)], 1024)])
def test_evict_of_many_short_heads_in_wide_tables(lens, max_pages):
    pool = U.Pool(lens, (8, 8, 64), BF, 16, max_pages=max_pages, spare=0)
    g = torch.Generator().manual_seed(8)
    w = torch.rand(pool.batch, 8, pool.cap, generator=g).to(DEV)
    T._check_evict(pool, w, None, 60, 3, 11, with_pos=False)


def test_the_most_sequences_and_heads():
    lens = [(3 * b) % 40 for b in range(1024)]
    T._check_attention(U.Pool(lens, (4, 2, 64), BF, 16), [b % 3 for b in range(1024)], True, seed=1)
    T._check_attention(U.Pool([40, 20], (1024, 1024, 64), BF, 16), [1, 1], False, seed=1)
