"""More of what the calls of the paged key-value cache refuse on the host: arrays that overlap what a call reads, widths beyond 31 bits.  No GPU."""
import pytest

import test_paged_refusals as R

P, ARG, SHAPE, WORKSPACE = R.P, R.ARG, R.SHAPE, R.WORKSPACE


@pytest.mark.parametrize("change", [
    dict(lens_out=7 * P), dict(lens_out=7 * P + 8), dict(lens_out=7 * P - 4), dict(seen=14 * P, seen_out=7 * P + 4), dict(lens_out=3 * P + 28),
    dict(seen=14 * P, seen_out=3 * P)])
def test_appends_to_arrays_that_they_read(change):
    """row_off has three entries at 7 P, the page table eight at 3 P."""
    rc, msg = R._append(**change)
    assert rc == ARG and "overlap" in msg, (rc, msg)


@pytest.mark.parametrize("change", [dict(lens_out=3 * P + 4), dict(weights_out=3 * P), dict(pos_out=3 * P), dict(weights_out=6 * P), dict(pos_out=6 * P - 4),
                                    dict(seen=14 * P, weights_out=14 * P), dict(lens_out=10 * P), dict(lens_out=11 * P + 4), dict(lens_out=12 * P),
                                    dict(lens_out=13 * P)])
def test_evictions_to_arrays_that_they_read_or_write(change):
    rc, msg = R._evict(**change)
    assert rc == ARG and "overlap" in msg, (rc, msg)


@pytest.mark.parametrize("change", [dict(weights_in=12 * P, weights_out=12 * P + 4), dict(weights_in=12 * P + 512, weights_out=12 * P)])
def test_weights_that_overlap_without_being_the_same(change):
    rc, msg = R._attention(**change)
    assert rc == ARG and "overlap" in msg, (rc, msg)


def test_weights_in_place_and_arrays_side_by_side_pass():
    """As far as the empty workspace."""
    assert R._attention(weights_in=12 * P, weights_out=12 * P)[0] == WORKSPACE
    per_slot = 2 * 4 * 64 * 4
    assert R._attention(weights_in=12 * P, weights_out=12 * P + per_slot)[0] == WORKSPACE
    assert R._evict(weights_out=10 * P + per_slot, pos_out=11 * P + per_slot, lens_out=6 * P + 8)[0] == WORKSPACE


@pytest.mark.parametrize("ld", [dict(ldq=1 << 24), dict(ldo=1 << 24)])
def test_rows_wider_than_31_bits_of_elements(ld):
    """2^24 heads of 128: a distance of rows that is smaller than a row is seen."""
    a = dict(n_heads=1 << 24, max_rows=1, ldq=1 << 31, ldo=1 << 31, workspace_bytes=0)
    a.update(ld)
    rc, msg = R._attention(**a)
    assert rc == ARG and "elements apart" in msg, (rc, msg)
