"""What the calls of the paged key-value cache refuse: found on the host before anything is launched, so it needs no GPU.  (The pointers
are made up; no call here gets as far as using one.)"""
import ctypes as C

import pytest

from paper_2603_05454_b200 import binding as B

P = 1 << 20           # a made-up, aligned address
ARG, SHAPE, WORKSPACE = -1, -2, -3


def _kv(**change):
    f = dict(k=P, v=2 * P, page_table=3 * P, status=None, page_stride=16 * 4 * 128, row_stride=4 * 128, head_stride=128, n_pages=10,
             page_size=16, max_pages=4, batch=2, n_kv_heads=4, head_dim=128, dtype=1)
    f.update(change)
    return B.PagedKV(*(f[n] for n, _ in B.PagedKV._fields_))


def _append(kv=None, **change):
    a = dict(k_new=4 * P, v_new=5 * P, ld=512, lens=6 * P, row_off=7 * P, max_rows=3, n_rows=5, lens_out=8 * P, weights=None, pos=None,
             seen=None, seen_out=None)
    a.update(change)
    e = C.create_string_buffer(256)
    return B.lib.lsp_paged_append(C.byref(kv or _kv()), *a.values(), None, e, 256), e.value.decode()


def _attention(kv=None, **change):
    a = dict(q=4 * P, ldq=1024, n_heads=8, lens=6 * P, row_off=7 * P, max_rows=3, n_rows=5, scale=0.1, out=5 * P, ldo=1024, lse=None,
             weights_in=None, weights_out=None, workspace=9 * P, workspace_bytes=0)
    a.update(change)
    e = C.create_string_buffer(256)
    return B.lib.lsp_paged_attention(C.byref(kv or _kv()), *a.values(), None, e, 256), e.value.decode()


def _evict(kv=None, **change):
    a = dict(weights=10 * P, pos=11 * P, lens=6 * P, seen=None, budget=32, n_sink=2, n_recent=8, weights_out=12 * P, pos_out=13 * P,
             lens_out=8 * P, workspace=9 * P, workspace_bytes=0)
    a.update(change)
    e = C.create_string_buffer(256)
    return B.lib.lsp_paged_evict(C.byref(kv or _kv()), *a.values(), None, e, 256), e.value.decode()


# Every call below would be refused for its empty workspace (attention, eviction) or its NULL lens_out (append) at the latest.
LAST = dict(append=lambda kv: _append(kv, lens_out=None), attention=_attention, evict=_evict)


@pytest.mark.parametrize("call", sorted(LAST))
@pytest.mark.parametrize("change,code,words", [
    (dict(k=None), ARG, "NULL"), (dict(v=None), ARG, "NULL"), (dict(dtype=2), ARG, "dtype"), (dict(head_dim=96), SHAPE, "head_dim"),
    (dict(n_pages=0), ARG, "positive"), (dict(page_size=0), ARG, "positive"), (dict(max_pages=0), ARG, "positive"),
    (dict(batch=0), ARG, "positive"), (dict(n_kv_heads=0), ARG, "positive"), (dict(batch=1025), SHAPE, "batch"),
    (dict(n_kv_heads=1025), SHAPE, "n_kv_heads"), (dict(max_pages=65537), SHAPE, "slots"), (dict(max_pages=1 << 30, page_size=1 << 30), SHAPE, "slots"),
    (dict(page_table=None, n_pages=7), ARG, "without a page table"), (dict(row_stride=516), ARG, "16 bytes"),
    (dict(head_stride=132), ARG, "16 bytes"), (dict(page_stride=8196), ARG, "16 bytes"), (dict(k=P + 8), ARG, "16 bytes"),
    (dict(row_stride=64), ARG, "smaller than a head"), (dict(head_stride=64), ARG, "smaller than a head"), (dict(page_stride=-8192), ARG, "smaller"),
    (dict(page_table=3 * P + 2), ARG, "misaligned"), (dict(status=3 * P + 1), ARG, "misaligned")])
def test_descriptions_that_no_call_takes(call, change, code, words):
    rc, msg = LAST[call](_kv(**change))
    assert rc == code and words in msg, (rc, msg)
    assert B.lib.lsp_paged_attention_workspace(C.byref(_kv(**change)), 8, 2, 0) == 0
    assert B.lib.lsp_paged_evict_workspace(C.byref(_kv(**change)), 32) == 0


@pytest.mark.parametrize("change,code,words", [
    (dict(lens=None), ARG, "NULL"), (dict(k_new=None), ARG, "NULL"), (dict(v_new=None), ARG, "NULL"), (dict(max_rows=0), ARG, "max_rows"),
    (dict(n_rows=-1), ARG, "n_rows"), (dict(row_off=None), ARG, "without row offsets"), (dict(ld=504), ARG, "elements apart"),
    (dict(ld=516), ARG, "aligned"), (dict(k_new=4 * P + 2), ARG, "aligned"), (dict(lens_out=6 * P), ARG, "overlap"),
    (dict(lens_out=6 * P + 4), ARG, "overlap"), (dict(seen=14 * P), ARG, "come together"), (dict(seen_out=14 * P), ARG, "come together"),
    (dict(seen=14 * P, seen_out=14 * P), ARG, "overlap"), (dict(seen=14 * P, seen_out=8 * P), ARG, "overlap"),
    (dict(seen=14 * P, seen_out=6 * P), ARG, "overlap"), (dict(weights=15 * P + 2), ARG, "misaligned")])
def test_appends(change, code, words):
    rc, msg = _append(**change)
    assert rc == code and words in msg, (rc, msg)


@pytest.mark.parametrize("change,code,words", [
    (dict(), WORKSPACE, "workspace of 0 bytes"), (dict(lens=None), ARG, "NULL"), (dict(q=None), ARG, "NULL"), (dict(out=None), ARG, "NULL"),
    (dict(workspace=None), ARG, "NULL"), (dict(n_heads=6), SHAPE, "query heads"), (dict(n_heads=0), SHAPE, "query heads"),
    (dict(scale=0.0), ARG, "scale"), (dict(scale=-1.0), ARG, "scale"), (dict(scale=float("nan")), ARG, "scale"), (dict(scale=float("inf")), ARG, "scale"),
    (dict(weights_in=12 * P), ARG, "weights_in"), (dict(ldq=1016), ARG, "elements apart"), (dict(ldo=1028), ARG, "aligned"),
    (dict(q=4 * P + 4), ARG, "aligned"), (dict(workspace=9 * P + 16), ARG, "256"), (dict(row_off=None), ARG, "without row offsets"),
    (dict(max_rows=-1), ARG, "max_rows"), (dict(lse=15 * P + 1), ARG, "misaligned")])
def test_attention(change, code, words):
    rc, msg = _attention(**change)
    assert rc == code and words in msg, (rc, msg)


def test_attention_of_more_work_than_one_call_takes():
    big = 1 << 40
    kv = _kv(batch=1024, n_kv_heads=1024, max_pages=65536, n_pages=1 << 30)
    rc, msg = _attention(kv, n_heads=1024, ldq=1024 * 128, ldo=1024 * 128, workspace_bytes=big)
    assert rc == SHAPE and "too large" in msg, (rc, msg)
    rc, msg = _attention(n_heads=8, max_rows=4097, n_rows=5, weights_out=12 * P, workspace_bytes=big)
    assert rc == SHAPE and "8192" in msg, (rc, msg)


@pytest.mark.parametrize("change,code,words", [
    (dict(), WORKSPACE, "workspace of 0 bytes"), (dict(weights=None), ARG, "NULL"), (dict(lens=None), ARG, "NULL"), (dict(lens_out=None), ARG, "NULL"),
    (dict(weights_out=None), ARG, "NULL"), (dict(workspace=None), ARG, "NULL"), (dict(pos_out=None), ARG, "pos_out"), (dict(budget=0), ARG, "budget"),
    (dict(n_sink=-1), ARG, "budget"), (dict(n_recent=-1), ARG, "budget"), (dict(n_recent=31), ARG, "budget"),
    (dict(n_sink=0x7fffffff, n_recent=0x7fffffff), ARG, "budget"), (dict(weights_out=10 * P), ARG, "overlap"), (dict(pos_out=11 * P + 256), ARG, "overlap"),
    (dict(lens_out=6 * P), ARG, "overlap"), (dict(seen=8 * P), ARG, "overlap"), (dict(pos_out=12 * P), ARG, "overlap"),
    (dict(workspace=9 * P + 128), ARG, "256"), (dict(lens=6 * P + 2), ARG, "misaligned")])
def test_evictions(change, code, words):
    rc, msg = _evict(**change)
    assert rc == code and words in msg, (rc, msg)


def test_workspace_sizes():
    ws = B.lib.lsp_paged_attention_workspace
    kv = _kv()
    plain = ws(C.byref(kv), 8, 6, 0)
    assert plain > 0 and plain % 256 == 0
    assert ws(C.byref(kv), 8, 6, 1) >= plain + 6 * 8 * 64 * 4                # a score per row, head and slot
    assert ws(C.byref(kv), 0, 6, 0) == 0 and ws(C.byref(kv), 8, -1, 0) == 0
    ev = B.lib.lsp_paged_evict_workspace
    assert ev(C.byref(kv), 32) >= 2 * 4 * (1 + 2 * 32) * 4                   # 32 of 64 slots move at most
    assert 0 < ev(C.byref(kv), 64) <= ev(C.byref(kv), 63) <= ev(C.byref(kv), 32)
    assert ev(C.byref(kv), 0) == 0


def test_a_message_buffer_is_optional():
    kv = _kv()
    assert B.lib.lsp_paged_append(C.byref(kv), *[None] * 2, 512, None, None, 1, 2, *[None] * 6, None, 0) == ARG
    assert B.lib.lsp_paged_append(None, *[None] * 2, 512, None, None, 1, 2, *[None] * 6, None, 0) == ARG
