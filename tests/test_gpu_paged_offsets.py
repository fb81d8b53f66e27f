"""Appends whose row offsets are partly out of range: the sequences with good offsets get every one of their rows, the others none."""
import numpy as np
import pytest
import torch

import paged_util as U
from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _check(heads, dtype, lens, row_off, n_rows, max_rows, bad=True):
    from paper_2603_05454_b200 import LSPError, PagedKVCache
    hq, hkv, dh = heads
    pool = U.Pool(lens, heads, dtype, 16, room=max_rows)
    width = hkv * dh
    new = torch.randn(n_rows, 2 * width, device=DEV).to(dtype)
    w = torch.full((len(lens), hkv, pool.cap), 7.0, device=DEV)
    pos = torch.full((len(lens), hkv, pool.cap), -7, dtype=torch.int32, device=DEV)
    seen = pool.lens + 3
    lens_out, seen_out = torch.zeros_like(seen), torch.zeros_like(seen)
    want_k, want_v, want_w, want_p, want_n = pool.k.clone(), pool.v.clone(), w.clone(), pos.clone(), list(lens)
    table, none = pool.table.tolist(), True
    for b, m in enumerate(lens):
        r0, r1 = row_off[b], row_off[b + 1]
        if not (0 <= r0 <= r1 <= n_rows and r1 - r0 <= max_rows):
            none = False
            continue
        for i in range(r1 - r0):
            p, s = table[b][(m + i) // 16], (m + i) % 16
            want_k[p, s] = new[r0 + i, :width].view(hkv, dh)
            want_v[p, s] = new[r0 + i, width:].view(hkv, dh)
            want_w[b, :, m + i] = 0
            want_p[b, :, m + i] = m + 3 + i
        want_n[b] = m + r1 - r0
    assert none != bad
    c = PagedKVCache(pool.k, pool.v, pool.table, n_heads=hq, max_rows=max_rows)
    c.append(new[:, :width], new[:, width:], pool.lens, lens_out, row_off=_ints(row_off), weights=w, pos=pos, seen=seen, seen_out=seen_out)
    if bad:
        with pytest.raises(LSPError) as e:
            c.check()
        assert "status 4)" in str(e.value)
    c.check()
    raw = torch.int16 if dtype == BF else torch.int32
    assert lens_out.tolist() == want_n and seen_out.tolist() == [n + 3 for n in want_n]
    assert torch.equal(w, want_w) and torch.equal(pos, want_p)
    assert torch.equal(pool.k.view(raw), want_k.view(raw)) and torch.equal(pool.v.view(raw), want_v.view(raw))


@pytest.mark.parametrize("heads,dtype", [((8, 4, 64), BF), ((32, 32, 128), F32)])        # (rows of 32 KB: more than a block holds at once)
@pytest.mark.parametrize("row_off,n_rows", [
    ([2, 1, 2], 5), ([0, 100, 2, 4, 6], 6), ([0, 2, -1, 2, 5], 5), ([5, 2, 0, 3, 4], 5), ([-1, 1, 3], 3), ([1, 2, 9, 3], 4),
    ([0, 3, 1, 3, 2, 4], 4),                                 # rows that two sequences name: appended to each
    ([4, 4, 0, 0, 2], 4), ([9, 8, 7, 6], 5), ([0, 2, 2 ** 31 - 1, -2 ** 31, 1], 4)])
def test_rows_of_good_sequences_beside_bad_offsets(heads, dtype, row_off, n_rows):
    _check(heads, dtype, [(11 * b) % 40 for b in range(len(row_off) - 1)], row_off, n_rows, 3)


@pytest.mark.parametrize("heads,dtype", [((1, 1, 64), BF), ((8, 4, 64), F32)])
@pytest.mark.parametrize("seed", [0, 1])
def test_many_sequences_and_rows(heads, dtype, seed):
    """As many rows that a block takes several; one offset in eight is wrong."""
    rng = np.random.default_rng(seed)
    rows = rng.integers(0, 25, 300)
    off = np.concatenate([[0], np.cumsum(rows)])
    n = int(off[-1])
    assert n > 2400
    _check(heads, dtype, [1] * 300, off.tolist(), n, 24, bad=False)
    at = rng.choice(301, 38, replace=False)
    off[at] += rng.integers(-60, 60, 38)
    _check(heads, dtype, [1] * 300, off.tolist(), n, 24)
