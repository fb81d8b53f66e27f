"""The paged key-value cache: append, attention of new rows with gathered weights, eviction, each against its definition in 64 bits, and a
run of them together next to a decoder."""
import math

import numpy as np
import pytest
import torch

import paged_util as U
from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
MHA, GQA, SMALL, ONE = (8, 8, 128), (28, 4, 128), (8, 4, 64), (1, 1, 64)


def _cache(pool, max_rows=1, weights=False, n_rows=None, table=True):
    from paper_2603_05454_b200 import PagedKVCache
    c = PagedKVCache(pool.k, pool.v, pool.table if table else None, n_heads=pool.heads[0], max_rows=max_rows, weights=weights, n_rows=n_rows)
    c.workspace[4096:].fill_(0xFF)                 # NaN bit patterns: no result depends on what nobody wrote
    return c


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _close(got, ref, tol, what):
    """|got - ref| <= tol element by element; equal infinities are equal."""
    got = got.double()
    bad = ~((got == ref) | ((got - ref).abs() <= tol))
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float((got - ref).abs().nan_to_num(1e30).max()):.3e}"


def _check_attention(pool, rows, ragged, weights=True, seed=0, scale=None, q_scale=2.0, max_rows=None, q=None):
    hq, hkv, dh = pool.heads
    n = sum(rows)
    max_rows = max_rows or max(max(rows), 1)
    row_off = _ints(np.concatenate([[0], np.cumsum(rows)])) if ragged else None
    behind = 2 if ragged else 0                    # rows behind the last sequence: nobody's
    g = torch.Generator().manual_seed(seed)
    qkv = (q_scale * torch.randn(n + behind, (hq + 2 * hkv) * dh, generator=g)).to(pool.dtype).to(DEV)
    q = qkv[:, : hq * dh] if q is None else q
    wide = torch.full((n + behind, hq * dh + 64), 7.0, dtype=pool.dtype, device=DEV)      # rows of out with something behind them
    out = wide[:, : hq * dh]
    lse = torch.full((n + behind, hq), 7.0, device=DEV)
    w_in = torch.rand(pool.batch, hkv, pool.cap, generator=g).to(DEV) if weights else None
    w_out = torch.full_like(w_in, 7.0) if weights else None
    c = _cache(pool, max_rows, weights, n + behind)
    c.attention(q, pool.lens, out, row_off=row_off, max_rows=max_rows if ragged else None, lse=lse, weights_in=w_in, weights_out=w_out, scale=scale)
    c.check()
    r_out, r_lse, r_w, size = U.attention(pool, q[:n], rows, w_in, scale)
    delta = U.relative_error(size, max(pool.lens_list), dh)
    v = max([float(pool.rows("v", b).abs().max()) for b in range(pool.batch) if pool.lens_list[b]] or [0.0])
    half = torch.finfo(pool.dtype).eps / 2         # the output's rounding; the bf16 weights' second part is off by half a step of half a step
    _close(out[:n], r_out, half * r_out.abs() + (2 * delta + (half ** 2 if pool.dtype == BF else 0)) * v * (1 + half), "out")
    _close(lse[:n], r_lse, 2 * delta + 2.0 ** -22 * r_lse.abs().nan_to_num(0, 0, 0), "lse")
    assert bool((wide[:, hq * dh:] == 7.0).all()) and bool((out[n:] == 7.0).all()) and bool((lse[n:] == 7.0).all())
    if weights:
        # what was added: each weight with its relative error; the sum of rows * group of them and of what was there, roundings of the sum
        for b, m in enumerate(pool.lens_list):
            added = r_w[b, :, :m] - w_in[b, :, :m].double()
            _close(w_out[b, :, :m], r_w[b, :, :m], 2 * delta * added + (max(rows) * hq // hkv + 1) * 2.0 ** -24 * r_w[b, :, :m], f"weights of sequence {b}")
            assert bool((w_out[b, :, m:] == 7.0).all())
    return out, lse, w_out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads", [MHA, GQA, SMALL, ONE])
@pytest.mark.parametrize("lens,page", [([1], 16), ([300], 16), ([0, 1, 15, 16, 17, 63, 64, 65], 16), ([129, 0, 1000, 64], 48), ([5, 700], 1), ([257, 256, 255], 256)])
def test_one_row_per_sequence(dtype, heads, lens, page):
    _check_attention(U.Pool(lens, heads, dtype, page, room=3), [1] * len(lens), False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,rows,max_rows", [
    (SMALL, [5, 0, 1, 3], 5),                # ten (row, head) pairs of a tile of sixteen; a sequence without rows
    (GQA, [4, 1, 3, 2], 4),                  # 28 pairs: two tiles, the second empty for a sequence of one row
    (MHA, [17, 16, 0, 33], 40),              # up to three tiles, a bound that nobody reaches
    ((7, 1, 64), [2, 2, 3, 0], 3)])
def test_blocks_of_rows(dtype, heads, rows, max_rows):
    _check_attention(U.Pool([90, 333, 0, 1025], heads, dtype, 32, room=1), rows, True, max_rows=max_rows, seed=3)


def test_equal_blocks_without_offsets():
    _check_attention(U.Pool([90, 333, 64], GQA, BF, 32), [3, 3, 3], False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,heads", [([30011], (7, 1, 128)), ([9000, 31, 20000, 0, 4097], (4, 2, 64))])
def test_long_sequences(dtype, lens, heads):
    _check_attention(U.Pool(lens, heads, dtype, 64), [1] * len(lens), False)


def test_many_sequences():
    lens = [(37 * b) % 190 for b in range(300)]
    _check_attention(U.Pool(lens, (2, 1, 64), BF, 16), [1] * 300, False)


@pytest.mark.parametrize("layout", ["heads", "mixed"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_other_orders_of_a_page(dtype, layout):
    _check_attention(U.Pool([100, 161], GQA, dtype, 32, layout=layout), [2, 1], True)


@pytest.mark.parametrize("scale,q_scale", [(0.5, 4.0), (1e-3, 1.0), (2.0, 8.0)])
def test_scales_from_flat_to_one_hot(scale, q_scale):
    _check_attention(U.Pool([500, 77], MHA, BF, 16), [1, 1], False, scale=scale, q_scale=q_scale)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 8, 9, 16, 17])
@pytest.mark.parametrize("scale,q_scale", [(None, 2.0), (1.0, 6.0)])
def test_fp32_groups_of_all_sizes(group, dh, scale, q_scale):
    """A kernel for each power of two of rows, full and not; maxima that rise late and far, too."""
    _check_attention(U.Pool([1, 77, 0, 640], (2 * group, 2, dh), F32, 16), [1] * 4, False, scale=scale, q_scale=q_scale, seed=group)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
def test_fp32_infinite_and_nan_rows_stay_with_their_head(group, dh):
    pool = U.Pool([100, 100], (4 * group, 4, dh), F32, 16)
    b0 = pool.table[0].long()
    pool.v[b0[1], 3, 2] = float("nan")
    pool.k[b0[2], 3, 1, 0] = float("inf")
    pool.k[b0[6], 4:, 3] = float("nan")            # the last page's slots behind the sequence
    pool.v[b0[6], 4:, 3] = float("nan")
    q = torch.rand(2, 4 * group * dh, device=DEV) + 0.5
    out = torch.empty_like(q)
    _cache(pool).attention(q, pool.lens, out)
    out = out.view(2, 4, group * dh)
    assert bool(out[0, 2].isnan().all()) and bool(out[0, 1].isnan().all())
    assert bool(out[0, 0].isfinite().all()) and bool(out[0, 3].isfinite().all()) and bool(out[1].isfinite().all())


def test_without_weights_the_same_bits():
    pool = U.Pool([700, 3, 64], GQA, BF, 16)
    a = _check_attention(pool, [1, 1, 1], False, weights=True)
    b = _check_attention(pool, [1, 1, 1], False, weights=False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_pages_shared_by_sequences():
    """Two sequences with one prefix: the same pages in both rows of the table."""
    pool = U.Pool([200, 150], GQA, BF, 16)
    pool.table[1, :8] = pool.table[0, :8]
    _check_attention(pool, [1, 1], False)


def test_weights_in_place_and_without_a_start():
    pool = U.Pool([200, 31], SMALL, BF, 16)
    q = torch.randn(2, 8 * 64, generator=torch.Generator().manual_seed(1)).to(BF).to(DEV)
    out, w, w2 = torch.empty_like(q), torch.rand(2, 4, pool.cap, device=DEV), torch.full((2, 4, pool.cap), 5.0, device=DEV)
    c = _cache(pool, 1, True)
    want = torch.empty_like(w)
    c.attention(q, pool.lens, out, weights_in=w, weights_out=want)
    c.attention(q, pool.lens, out, weights_out=w2)
    c.attention(q, pool.lens, out, weights_in=w, weights_out=w)
    for b, n in enumerate(pool.lens_list):
        assert torch.equal(w[b, :, :n], want[b, :, :n])
        assert bool((w2[b, :, n:] == 5).all())
        assert abs(float(w2[b, :, :n].sum()) - 8) < 1e-4               # eight query heads, weights that sum to one
    c.check()


def test_infinite_and_nan_rows_stay_with_their_head():
    pool = U.Pool([100, 100], (4, 4, 64), BF, 16)
    b0 = pool.table[0].long()
    pool.v[b0[1], 3, 2] = float("nan")
    pool.k[b0[2], 3, 1, 0] = float("inf")
    q = torch.rand(2, 256, device=DEV).to(BF) + 0.5
    out = torch.empty_like(q)
    c = _cache(pool)
    c.attention(q, pool.lens, out)
    out = out.view(2, 4, 64)
    assert bool(out[0, 2].isnan().all()) and bool(out[0, 1].isnan().all())
    assert bool(out[0, 0].isfinite().all()) and bool(out[0, 3].isfinite().all()) and bool(out[1].isfinite().all())


def test_a_row_whose_scores_are_all_minus_infinity_is_empty():
    pool = U.Pool([70], (2, 1, 64), BF, 16)
    pool.k[pool.table[0].long()[:5], :, 0, 0] = float("-inf")
    q = torch.zeros(1, 128, dtype=BF, device=DEV)
    q[0, 0] = 1.0
    q[0, 64] = -1.0                                                # the other head: all +inf, as the formula says NaN
    out, lse, w = torch.full_like(q, 7.0), torch.empty(1, 2, device=DEV), torch.ones(1, 1, pool.cap, device=DEV)
    c = _cache(pool, 1, True)
    c.attention(q, pool.lens, out, lse=lse, weights_in=w, weights_out=w)
    assert bool((out[0, :64] == 0).all()) and float(lse[0, 0]) == -math.inf
    assert bool(out[0, 64:].isnan().all())


def test_offsets_beyond_32_bits():
    """Pages more than 2^31 bytes, and in all more than 2^32, apart."""
    heads, page = (4, 2, 128), 16
    stride = (1 << 31) // 2 + 4096                    # elements: 2 GB and a bit
    base = torch.empty(2 * stride + 2 * page * 256 + 64, dtype=BF, device=DEV)
    shape, strides = (3, page, 2, 128), (stride, 256, 128, 1)
    pool = U.Pool([40], heads, BF, page, spare=0)
    k, v = (torch.as_strided(base, shape, strides, storage_offset=o) for o in (0, page * 256))
    k.copy_(pool.k)
    v.copy_(pool.v)
    pool.k, pool.v = k, v
    _check_attention(pool, [1], False)
    # an eviction and an append over the same distances
    kv = [pool.rows(x, 0).clone() for x in "kv"]
    w = torch.rand(1, 2, pool.cap, device=DEV)
    w_out, lens_out = torch.empty_like(w), torch.zeros(1, dtype=torch.int32, device=DEV)
    c = _cache(pool)
    c.evict(w, pool.lens, 20, w_out, lens_out)
    new = torch.randn(2, 512, device=DEV).to(BF)
    lens2 = torch.zeros_like(lens_out)
    c.append(new[:, :256], new[:, 256:], _ints([40]), lens2)
    c.check()
    for h in range(2):
        place = U.evict(w[0, h].cpu(), range(40), 40, 20, 0, 0, 40)
        for x, full in zip("kv", kv):
            assert torch.equal(pool.rows(x, 0)[:20, h], full[place, h])
    assert torch.equal(pool.rows("k", 0, 42)[40:].reshape(2, 256), new[:, :256].double())
    assert torch.equal(pool.rows("v", 0, 42)[40:].reshape(2, 256), new[:, 256:].double())


def test_the_same_bits_every_time_and_whatever_else_is_in_the_batch_is_right():
    pool = U.Pool([3000, 1, 777, 64, 2049], GQA, BF, 64)
    q = torch.randn(5, 28 * 128, device=DEV).to(BF)
    c = _cache(pool, 1, True)
    outs = []
    for _ in range(3):
        out, w = torch.empty_like(q), torch.zeros(5, 4, pool.cap, device=DEV)
        c.attention(q, pool.lens, out, weights_in=torch.zeros_like(w), weights_out=w)
        outs.append((out, w))
    for out, w in outs[1:]:
        assert torch.equal(out, outs[0][0]) and torch.equal(w, outs[0][1])


# ---- what only the device sees ------------------------------------------------------------------------------------------

def _raises(c, bits):
    from paper_2603_05454_b200 import LSPError
    with pytest.raises(LSPError) as e:
        c.check()
    assert e.value.code == -4 and f"status {bits})" in str(e.value), str(e.value)
    c.check()                                        # cleared


def test_bad_pages_get_no_weight_and_a_status():
    pool = U.Pool([100, 50], SMALL, BF, 16)
    good = pool.table.clone()
    q = torch.randn(2, 512, device=DEV).to(BF)
    out, out2, w = torch.empty_like(q), torch.empty_like(q), torch.zeros(2, 4, pool.cap, device=DEV)
    c = _cache(pool, 1, True)
    c.attention(q, pool.lens, out)
    c.check()
    pool.table[0, 2] = pool.k.shape[0]
    pool.table[0, 4] = -1
    pool.table[1, 5] = -7                            # behind the length: not looked at
    c.attention(q, pool.lens, out2, weights_out=w)
    _raises(c, 2)
    assert torch.equal(out[1], out2[1]) and bool(out2.isfinite().all()) and not torch.equal(out[0], out2[0])
    assert bool((w[0, :, 32:48] == 0).all()) and bool((w[0, :, 64:80] == 0).all()) and bool((w[0, :, 48:64] > 0).all())
    pool.table[0] = pool.k.shape[0]                  # no page at all: nothing seen
    c.attention(q, pool.lens, out2, weights_out=w)
    _raises(c, 2)
    assert bool((out2[0] == 0).all()) and bool((w[0, :, :100] == 0).all()) and torch.equal(out[1], out2[1])
    pool.table.copy_(good)
    c.attention(q, pool.lens, out2)
    c.check()
    assert torch.equal(out, out2)


def test_bad_lengths_are_clamped():
    pool = U.Pool([64, 48], SMALL, BF, 16, max_pages=4)
    q = torch.randn(2, 512, device=DEV).to(BF)
    want, got = torch.empty_like(q), torch.empty_like(q)
    c = _cache(pool)
    c.attention(q, _ints([64, 0]), want)
    c.check()
    c.attention(q, _ints([1000, -5]), got)
    _raises(c, 1)
    assert torch.equal(want, got)
    w = torch.rand(2, 4, pool.cap, device=DEV)
    w_out, lens_out = torch.empty_like(w), _ints([9, 9])
    before = pool.rows("k", 1).clone()
    c.evict(w, _ints([1 << 30, -1]), 40, w_out, lens_out)
    _raises(c, 1)
    assert lens_out.tolist() == [40, 0] and torch.equal(pool.rows("k", 1), before)


@pytest.mark.parametrize("row_off", [[0, 3, 2], [-1, 1, 2], [0, 1, 9], [2, 1, 2], [0, 4, 5]])
def test_bad_row_offsets_leave_their_sequence_alone(row_off):
    """Five rows, at most three of a sequence: sequences whose offsets are no good have no rows, the other's rows are right."""
    pool = U.Pool([64, 48], SMALL, BF, 16, room=16)
    good = [0 <= row_off[b] <= row_off[b + 1] <= 5 and row_off[b + 1] - row_off[b] <= 3 for b in range(2)]
    q = torch.randn(5, 512, device=DEV).to(BF)
    out = torch.full_like(q, 7.0)
    c = _cache(pool, 3)
    c.attention(q, pool.lens, out, row_off=_ints(row_off))
    _raises(c, 4)
    for b in range(2):
        if good[b]:
            rows = slice(row_off[b], row_off[b + 1])
            one = U.attention(pool, q[rows], [row_off[b + 1] - row_off[b] if i == b else 0 for i in range(2)])[0]
            assert float((out[rows].double() - one).abs().max() if one.numel() else 0) < 0.02
            out[rows] = 7.0
    assert bool((out == 7.0).all())
    kv = torch.randn(5, 512, device=DEV).to(BF)
    before = pool.k.clone()
    lens_out = _ints([0, 0])
    c.append(kv[:, :256], kv[:, 256:], pool.lens, lens_out, row_off=_ints(row_off))
    _raises(c, 4)
    assert lens_out.tolist() == [n + (row_off[b + 1] - row_off[b] if good[b] else 0) for b, n in enumerate(pool.lens_list)]
    if not any(good):
        assert torch.equal(pool.k.view(torch.int16), before.view(torch.int16))


# ---- append --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,lens,rows,page,layout", [
    (MHA, [0], [1], 16, "slots"), (GQA, [15, 16, 17, 0], [1, 1, 1, 1], 16, "heads"), (SMALL, [5, 0, 30], [0, 40, 3], 16, "slots"),
    ((32, 32, 128), [0, 7], [70, 33], 64, "slots"), (ONE, [3, 0, 0, 2], [0, 0, 5, 0], 1, "mixed"), (SMALL, [1] * 300, [b % 3 for b in range(300)], 4, "slots")])
@pytest.mark.parametrize("ragged", [True, False])
def test_append(dtype, heads, lens, rows, page, layout, ragged):
    if not ragged:
        rows = [max(rows)] * len(rows)
    hq, hkv, dh = heads
    pool = U.Pool(lens, heads, dtype, page, room=max(rows), layout=layout)
    n, width = sum(rows), hkv * dh
    behind = 2 if ragged else 0
    new = torch.randn(n + behind, 2 * width + 64, device=DEV).to(dtype)
    row_off = _ints(np.concatenate([[0], np.cumsum(rows)])) if ragged else None
    w = torch.full((len(lens), hkv, pool.cap), 7.0, device=DEV)
    pos = torch.full((len(lens), hkv, pool.cap), -7, dtype=torch.int32, device=DEV)
    seen = pool.lens + 3
    lens_out, seen_out = torch.zeros_like(seen), torch.zeros_like(seen)
    want_k, want_v, want_w, want_p = pool.k.clone(), pool.v.clone(), w.clone(), pos.clone()
    at, table = 0, pool.table.tolist()
    for b, (m, r) in enumerate(zip(lens, rows)):
        for i in range(r):
            p, s = table[b][(m + i) // page], (m + i) % page
            want_k[p, s] = new[at, :width].view(hkv, dh)
            want_v[p, s] = new[at, width:2 * width].view(hkv, dh)
            want_w[b, :, m + i] = 0
            want_p[b, :, m + i] = m + 3 + i
            at += 1
    c = _cache(pool, max(rows))
    c.append(new[:, :width], new[:, width:2 * width], pool.lens, lens_out, row_off=row_off, weights=w, pos=pos, seen=seen, seen_out=seen_out)
    c.check()
    raw = torch.int16 if dtype == BF else torch.int32
    assert torch.equal(pool.k.view(raw), want_k.view(raw)) and torch.equal(pool.v.view(raw), want_v.view(raw))
    assert torch.equal(w, want_w) and torch.equal(pos, want_p)
    assert lens_out.tolist() == [m + r for m, r in zip(lens, rows)] and seen_out.tolist() == [m + 3 + r for m, r in zip(lens, rows)]
    # without weights, positions and seen: the same rows
    pool.k.fill_(1.0)
    pool.v.fill_(2.0)
    before = [(m, r) for m, r in zip(lens, rows)]
    c.append(new[:, :width], new[:, width:2 * width], pool.lens, lens_out, row_off=row_off)
    at = 0
    for b, (m, r) in enumerate(before[:8]):
        assert torch.equal(pool.rows("k", b, m + r)[m:].reshape(r, width), new[at:at + r, :width].double())
        at += r


def test_append_past_the_last_page_and_to_bad_pages():
    pool = U.Pool([30, 16, 0], SMALL, BF, 16, max_pages=2, spare=0)
    pool.table[1, 1] = 99
    new = torch.randn(12, 512, device=DEV).to(BF)
    lens_out, pos = _ints([0, 0, 0]), torch.full((3, 4, 32), -1, dtype=torch.int32, device=DEV)
    k1 = pool.rows("k", 0).clone()
    c = _cache(pool, 4)
    c.append(new[:, :256], new[:, 256:], pool.lens, lens_out, pos=pos)
    _raises(c, 3)
    assert lens_out.tolist() == [32, 20, 4]
    assert torch.equal(pool.rows("k", 0), k1) and torch.equal(pool.rows("k", 0, 32)[30:].reshape(2, 256), new[:2, :256].double())
    assert torch.equal(pool.rows("v", 2, 4).reshape(4, 256), new[8:, 256:].double())
    assert pos[0, 0, 30:].tolist() == [30, 31] and bool((pos[1] == -1).all()) and pos[2, 3, :5].tolist() == [0, 1, 2, 3, -1]


# ---- eviction ------------------------------------------------------------------------------------------------------------

def _check_evict(pool, w, pos, budget, sink=0, recent=0, seen=None, with_pos=True):
    hq, hkv, dh = pool.heads
    raw = torch.int16 if pool.dtype == BF else torch.int32
    k, v = pool.k.clone(), pool.v.clone()
    w_out, p_out = torch.full_like(w, 7.0), torch.full(w.shape, -7, dtype=torch.int32, device=DEV)
    lens_out = torch.zeros_like(pool.lens)
    c = _cache(pool)
    c.evict(w, pool.lens, budget, w_out, lens_out, n_sink=sink, n_recent=recent, pos=pos if with_pos else None, pos_out=p_out, seen=seen)
    c.check()
    assert lens_out.tolist() == [min(n, budget) for n in pool.lens_list]
    want_k, want_v, want_w, want_p = k.clone(), v.clone(), torch.full_like(w, 7.0), torch.full_like(p_out, -7)
    table = pool.table.long()
    for b, n in enumerate(pool.lens_list):
        s = n if seen is None else int(seen[b])
        for h in range(hkv):
            p = pos[b, h] if with_pos else torch.arange(pool.cap, dtype=torch.int32, device=DEV)
            place = torch.tensor(U.evict(w[b, h].cpu(), p.cpu(), n, budget, sink, recent, s), dtype=torch.long, device=DEV)
            to = torch.arange(len(place), device=DEV)
            want_w[b, h, :len(place)] = w[b, h, place]
            want_p[b, h, :len(place)] = p[place]
            for new, old in ((want_k, k), (want_v, v)):
                new[table[b, to // pool.page], to % pool.page, h] = old[table[b, place // pool.page], place % pool.page, h]
    assert torch.equal(p_out, want_p)
    assert torch.equal(w_out.view(torch.int32), want_w.view(torch.int32))
    assert torch.equal(pool.k.view(raw), want_k.view(raw)) and torch.equal(pool.v.view(raw), want_v.view(raw))


def _weights(pool, seed, ties=True):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(2 * torch.randn(pool.batch, pool.heads[1], pool.cap, generator=g))
    if ties:
        w = torch.where(torch.rand(w.shape, generator=g) < 0.3, torch.round(w), w)
    pos = torch.full(w.shape, 1 << 20, dtype=torch.int32)
    for b, n in enumerate(pool.lens_list):
        for h in range(pool.heads[1]):
            pos[b, h, :n] = torch.randperm(n + 5, generator=g)[:n].to(torch.int32)
    return w.to(DEV), pos.to(DEV)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,lens,budget,sink,recent,page", [
    (SMALL, [100, 40, 41, 0, 39], 40, 3, 10, 16), (GQA, [257, 1000], 130, 0, 0, 48), (MHA, [64, 65], 64, 4, 60, 16), (ONE, [1, 2, 3], 1, 0, 1, 1),
    (ONE, [33], 32, 32, 0, 16), ((2, 2, 64), [2047, 1025], 1024, 4, 64, 64)])
def test_evict(dtype, heads, lens, budget, sink, recent, page):
    pool = U.Pool(lens, heads, dtype, page, room=2)
    w, pos = _weights(pool, 5)
    _check_evict(pool, w, pos, budget, sink, recent, seen=pool.lens + 5)


@pytest.mark.parametrize("layout", ["heads", "mixed"])
def test_evict_from_other_orders_of_a_page(layout):
    pool = U.Pool([100, 77], GQA, BF, 32, layout=layout)
    w, pos = _weights(pool, 6)
    _check_evict(pool, w, pos, 50, 2, 10)


@pytest.mark.parametrize("n,budget", [(40000, 8192), (33000, 32999), (70001, 100)])
def test_evict_from_a_long_sequence(n, budget):
    pool = U.Pool([n], (2, 2, 64), BF, 64)
    w, pos = _weights(pool, 7)
    _check_evict(pool, w, pos, budget, 5, 50)


def test_evict_from_more_slots_than_are_kept_on_chip():
    pool = U.Pool([400001], (1, 1, 64), BF, 64)
    w, pos = _weights(pool, 17)
    _check_evict(pool, w, pos, 150000, 5, 5000)


@pytest.mark.parametrize("budget", [40, 75])
def test_evict_of_many_heads(budget):
    pool = U.Pool([70 + b % 9 for b in range(40)], (8, 8, 64), BF, 16)
    w, pos = _weights(pool, 18)
    _check_evict(pool, w, pos, budget, 3, 11)


@pytest.mark.parametrize("values", [[1.0], [0.0, 2.0]])
def test_ties_over_a_cluster(values):
    pool = U.Pool([20000], (2, 2, 64), BF, 64)
    _, pos = _weights(pool, 19)
    w = torch.tensor(values)[torch.randint(len(values), (1, 2, pool.cap), generator=torch.Generator().manual_seed(3))].to(DEV)
    _check_evict(pool, w, pos, 15000, 3, 11)


def test_evict_without_positions_goes_by_slots():
    pool = U.Pool([300, 20], SMALL, BF, 16)
    w, _ = _weights(pool, 8)
    _check_evict(pool, w, None, 100, 4, 20, with_pos=False)


@pytest.mark.parametrize("values", [[0.0], [1.0, 1.0, 2.0], [0.0, -0.0], [math.nan, 1.0], [math.inf, 1.0, -math.inf, math.nan], [-1.0, -2.0, 0.0],
                                    [1e-45, 0.0, 3e-39], [1.0, 1.0 + 2 ** -23]])
def test_ties_and_odd_weights(values):
    pool = U.Pool([200, 90], SMALL, BF, 16)
    _, pos = _weights(pool, 9)
    g = torch.Generator().manual_seed(2)
    w = torch.tensor(values)[torch.randint(len(values), (2, 4, pool.cap), generator=g)].to(DEV)
    _check_evict(pool, w, pos, 64, 3, 9, seen=pool.lens + 5)


def test_positions_that_come_twice_leave_the_budget_exact():
    pool = U.Pool([200], SMALL, BF, 16)
    w = torch.ones(1, 4, pool.cap, device=DEV)
    pos = (torch.arange(pool.cap, device=DEV, dtype=torch.int32) // 3).expand(1, 4, -1).contiguous()
    _check_evict(pool, w, pos, 64)
    _check_evict(pool, w, pos, 64, 60, 4, seen=_ints([1]))       # more protected slots than the budget holds: the lower positions


# ---- together ------------------------------------------------------------------------------------------------------------

def test_captured_calls_follow_their_lengths():
    """One step (append, attention, eviction) captured once and replayed on other rows, lengths and pages; an eager object beside it."""
    pool = U.Pool([70, 33], SMALL, BF, 16, room=20)
    other = U.Pool([50, 60], SMALL, BF, 16, seed=4)
    eager = _cache(other)
    c = _cache(pool, 1, True)
    kvq = torch.randn(2, 1024, device=DEV).to(BF)
    q, kn, vn = kvq[:, :512], kvq[:, 512:768], kvq[:, 768:]
    lens, lens2, lens3 = pool.lens, _ints([0, 0]), _ints([0, 0])
    seen, seen2 = pool.lens.clone(), _ints([0, 0])
    w, w2, w3 = (torch.zeros(2, 4, pool.cap, device=DEV) for _ in range(3))
    pos = torch.arange(pool.cap, device=DEV, dtype=torch.int32).expand(2, 4, -1).contiguous()
    pos2, out, oq, oo = torch.zeros_like(pos), torch.empty(2, 512, dtype=BF, device=DEV), kvq[:, :512].clone(), torch.empty(2, 512, dtype=BF, device=DEV)

    def step(cache, stream=None):
        cache.append(kn, vn, lens, lens2, weights=w, pos=pos, seen=seen, seen_out=seen2, stream=stream)
        cache.attention(q, lens2, out, weights_in=w, weights_out=w2, stream=stream)
        cache.evict(w2, lens2, 40, w3, lens3, n_sink=2, n_recent=5, pos=pos, pos_out=pos2, seen=seen2, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        keep = [t.clone() for t in (pool.k, pool.v, w, pos)]
        step(c)                                       # once eagerly on the capturing stream
        for t, x in zip((pool.k, pool.v, w, pos), keep):
            t.copy_(x)
        with torch.cuda.graph(graph, stream=side):
            step(c)
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(3):
        kvq.copy_(torch.randn(2, 1024, generator=torch.Generator().manual_seed(turn)).to(BF))
        eager.attention(oq, other.lens, oo)
        graph.replay()
        got = [t.clone() for t in (out, w3, pos2, lens3, seen2, pool.k, pool.v)]
        for t, x in zip((pool.k, pool.v, w, pos), keep):
            t.copy_(x)
        step(c)
        for a, b in zip(got, (out, w3, pos2, lens3, seen2, pool.k, pool.v)):
            assert torch.equal(a.view(torch.int16) if a.dtype == BF else a, b.view(torch.int16) if b.dtype == BF else b)
        # the next turn goes on from here
        lens.copy_(lens3)
        seen.copy_(seen2)
        n = [int(x) for x in lens3]
        w.copy_(w3)
        pos.copy_(pos2)
        keep = [t.clone() for t in (pool.k, pool.v, w, pos)]
    assert lens.tolist() == [40, 36] and seen.tolist() == [73, 36]
    c.check()
    eager.check()
    assert bool(oo.isfinite().all())


def test_two_streams_with_an_object_each():
    pool = U.Pool([900, 333], GQA, BF, 16)
    q = [torch.randn(2, 28 * 128, device=DEV).to(BF) for _ in range(2)]
    want = [torch.empty_like(x) for x in q]
    ref = _cache(pool)
    for x, o in zip(q, want):
        ref.attention(x, pool.lens, o)
    streams, caches, outs = [torch.cuda.Stream() for _ in range(2)], [_cache(pool) for _ in range(2)], [torch.empty_like(x) for x in q]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, c, x, o in zip(streams, caches, q, outs):
            c.attention(x, pool.lens, o, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_two_threads_with_an_object_each():
    """Calls of unlike shapes from two host threads, each on its own stream: what a launch needs is set per call."""
    import threading
    pools = [U.Pool([900, 333], GQA, BF, 16), U.Pool([50, 700, 1], (8, 8, 128), BF, 32, seed=1)]
    q = [torch.randn(p.batch, p.heads[0] * 128, device=DEV).to(BF) for p in pools]
    want, got, caches = [torch.empty_like(x) for x in q], [torch.empty_like(x) for x in q], [_cache(p, 1, True) for p in pools]
    w = [torch.rand(p.batch, p.heads[1], p.cap, device=DEV) for p in pools]
    for c, p, x, o in zip(caches, pools, q, want):
        c.attention(x, p.lens, o)
    torch.cuda.synchronize()
    failed = []

    def work(i):
        try:
            s = torch.cuda.Stream()
            w_out, lens_out = torch.empty_like(w[i]), torch.empty_like(pools[i].lens)
            for _ in range(40):
                caches[i].attention(q[i], pools[i].lens, got[i], stream=s)
                caches[i].evict(w[i], pools[i].lens, 2000, w_out, lens_out, stream=s)      # (nothing to evict)
            s.synchronize()
        except Exception as e:
            failed.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed and all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_rows_at_all():
    pool = U.Pool([40, 7], SMALL, BF, 16)
    c = _cache(pool, 2, True)
    w, w_out = torch.rand(2, 4, pool.cap, device=DEV), torch.full((2, 4, pool.cap), 7.0, device=DEV)
    empty = torch.empty(0, 512, dtype=BF, device=DEV)
    c.attention(empty, pool.lens, empty, row_off=_ints([0, 0, 0]), weights_in=w, weights_out=w_out)
    c.attention(empty, pool.lens, empty, row_off=_ints([0, 0, 0]))
    lens_out = _ints([0, 0])
    c.append(empty[:, :256], empty[:, 256:], pool.lens, lens_out, row_off=_ints([0, 0, 0]))
    c.check()
    for b, n in enumerate(pool.lens_list):
        assert torch.equal(w_out[b, :, :n], w[b, :, :n]) and bool((w_out[b, :, n:] == 7).all())
    assert lens_out.tolist() == [40, 7]


def test_calls_that_the_object_refuses():
    from paper_2603_05454_b200 import LSPError, PagedKVCache
    pool = U.Pool([40, 7], SMALL, BF, 16)
    c = _cache(pool, 1)
    q, out = torch.zeros(2, 512, dtype=BF, device=DEV), torch.zeros(2, 512, dtype=BF, device=DEV)
    w = torch.zeros(2, 4, pool.cap, device=DEV)
    bad = [dict(q=q.float()), dict(q=q[:, :256]), dict(q=q.cpu()), dict(q=q.t()), dict(q=q[:1]), dict(out=out[:1]), dict(lens=pool.lens.long()),
           dict(lens=pool.lens[:1]), dict(lse=torch.zeros(2, 7, device=DEV)), dict(row_off=_ints([0, 2])), dict(weights_out=w[:, :, :-1])]
    for change in bad:
        a = dict(q=q, lens=pool.lens, out=out)
        a.update(change)
        with pytest.raises(ValueError):
            c.attention(a.pop("q"), a.pop("lens"), a.pop("out"), **a)
    for code, call in [(-3, lambda: c.attention(q, pool.lens, out, weights_out=w)),                   # made without room for weights
                       (-1, lambda: c.attention(q, pool.lens, out, scale=-1.0)), (-1, lambda: c.evict(w, pool.lens, 4, w.clone(), pool.lens.clone(), n_recent=5)),
                       (-1, lambda: c.evict(w, pool.lens, 4, w, pool.lens.clone())), (-1, lambda: c.append(q[:, :256], q[:, 256:], pool.lens, pool.lens))]:
        with pytest.raises(LSPError) as e:
            call()
        assert e.value.code == code
    for k, v, t in [(pool.k, pool.v[:, :, :, :32], pool.table), (pool.k, pool.v.float(), pool.table), (pool.k.half(), pool.v.half(), pool.table),
                    (pool.k[0], pool.v[0], pool.table), (pool.k, pool.v, pool.table.long()), (pool.k, pool.v, pool.table[0])]:
        with pytest.raises(ValueError):
            PagedKVCache(k, v, t, n_heads=8)
    with pytest.raises(LSPError):
        PagedKVCache(pool.k[:, :, :, :32], pool.v[:, :, :, :32], pool.table, n_heads=8)                 # heads of 32
    c.check()


def test_next_to_a_decoder():
    """The cache that a decode leaves behind, taken as pages in place (a sequence a page): the attention equals lsp_op_attention's, rows are appended to
    the decoder's own planes, and after an eviction the attention is that over the kept rows."""
    import lsp_synth as S
    from paper_2603_05454_b200 import LSPDecoder, PagedKVCache, SchedCfg
    sh = S.ModelShape(2, 512, 4, 2, 128, 1024, 4096, dtype="bf16", head_scale=1.5, w_std=0.044)
    B, P, G = 2, 40, 24
    dec = LSPDecoder(sh, S.make_weights(sh, 0, device=DEV), SchedCfg(tau=0.05), B, 128, device=DEV)
    tokens = torch.zeros(B, P + G, dtype=torch.int32, device=DEV)
    tokens[:, :P] = S.make_prompt(B, P, sh, 0).to(DEV)
    n, recs = 0, []
    dec.begin(tokens, [P, P - 7], [G, G])
    n, recs = dec.generate(max_recs=2 * G * B)
    done = [sum(r["L_commit"] for r in recs[b::B] if r["n_before"]) for b in range(B)]
    assert done == [G, G]
    # the block committed last is still pending: the cache holds all rows ahead of it
    last = [[r["L_commit"] for r in recs[b::B] if r["n_before"]][-1] for b in range(B)]
    lens = [P + G - last[0], P - 7 + G - last[1]]
    planes = dec.kv_view()[1]                                 # layer 1: [K|V][sequence][position][head][i]
    cache = PagedKVCache(planes[0], planes[1], n_heads=4, batch=B, max_rows=3, weights=True)
    assert cache.max_pages == 1 and cache.capacity == 128
    rows = [3, 2]
    q = S.normal((5, 512), 3, 1, 1.0, BF, DEV)
    kn, vn = S.normal((5, 256), 3, 2, 1.0, BF, DEV), S.normal((5, 256), 3, 3, 1.0, BF, DEV)
    want = torch.empty_like(q)
    dec.op_attention(1, q, kn, vn, want, lens, rows)
    row_off, ln, ln2, ln3 = _ints([0, 3, 5]), _ints(lens), _ints([0, 0]), _ints([0, 0])
    w, w2, w3 = (torch.zeros(B, 2, 128, device=DEV) for _ in range(3))
    pos = torch.arange(128, device=DEV, dtype=torch.int32).expand(B, 2, -1).contiguous()
    pos2 = torch.zeros_like(pos)
    cache.append(kn, vn, ln, ln2, row_off=row_off, weights=w, pos=pos)
    got = torch.empty_like(q)
    cache.attention(q, ln2, got, row_off=row_off, weights_in=w, weights_out=w2)
    # both within half a bf16 step of the formula (and the other kernel's bf16 weights: another half): a step of the larger
    a, b = got.double(), want.double()
    assert float(((a - b).abs() - 2 * 2.0 ** -8 * torch.maximum(a.abs(), b.abs())).max()) < 4e-3
    total = [lens[0] + 3, lens[1] + 2]
    assert ln2.tolist() == total
    k, v = planes[0].double().clone(), planes[1].double().clone()
    cache.evict(w2, ln2, 30, w3, ln3, n_sink=1, n_recent=4, pos=pos, pos_out=pos2)
    cache.attention(q, ln3, got, row_off=row_off)
    cache.check()
    assert ln3.tolist() == [30, 30]
    at = 0
    for s in range(B):
        for h in range(4):
            keep = pos2[s, h // 2, :30].long()
            assert 0 in keep.tolist() and all(p in keep.tolist() for p in range(total[s] - 4, total[s]))
            qq = q[at:at + rows[s], h * 128:(h + 1) * 128].double()
            p = torch.softmax(qq @ k[s, keep, h // 2].T / 128 ** 0.5, -1)
            r = p @ v[s, keep, h // 2]
            g = got[at:at + rows[s], h * 128:(h + 1) * 128].double()
            assert float(((g - r).abs() - 2.0 ** -8 * r.abs()).max()) < 1e-3
        at += rows[s]
    dec.close()
