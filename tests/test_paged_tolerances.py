"""What the checks of long sequences notice: mistakes planted in the definition, on the CPU."""
import pytest
import torch

import paged_long as L


def _half(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,dh", [(30011, 128), (12345, 64)])
def test_a_lost_or_repeated_group_of_slots_shows_in_counts(dtype, n, dh):
    v = L.counted_values(n, dh).double()
    ref = v.mean(0)
    tol = L.counted_tolerance(ref, _half(dtype))
    rounded = ref.to(dtype).double()
    assert bool(((rounded - ref).abs() <= tol).all())
    for at in list(range(0, n, 16 * 97)) + [(n - 1) // 16 * 16]:
        part = v[at:at + 16]
        if len(part) < 16 and dtype == torch.bfloat16:
            continue                                            # (a last group of a few slots is less than bf16 resolves: lse shows it)
        lost, twice = (v.sum(0) - part.sum(0)) / (n - len(part)), (v.sum(0) + part.sum(0)) / n
        swapped = (v.sum(0) - part.sum(0) + v[(at + 16 * 31) % (n - 32):][:len(part)].sum(0)) / n
        for wrong in (lost, twice, swapped):
            assert bool(((wrong - ref).abs() > tol).any()), at
    # one slot less shows in the log of the sum
    assert abs(float(torch.log(torch.tensor(n, dtype=torch.float64)) - torch.log(torch.tensor(n - 1, dtype=torch.float64)))) > 8 * 2.0 ** -22 * 10.4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,dh", [(30011, 128), (20000, 64)])
def test_a_lost_chunk_shows_in_random_rows(dtype, n, dh):
    g = torch.Generator().manual_seed(n)
    q = (2 * torch.randn(4, dh, generator=g)).to(dtype)
    k, v = (torch.randn(n, dh, generator=g).to(dtype) for _ in range(2))
    out, magnitude, _, size, p = L.reference(q, k, v, dh ** -0.5)
    tol = L.tolerance(out, magnitude, size, dh, _half(dtype))
    assert bool(((out.to(dtype).double() - out).abs() <= tol).all())
    for at in range(0, n - 64, 64 * 29):
        keep = torch.ones(n, dtype=torch.bool)
        keep[at:at + 64] = False
        pk = p[:, keep] / p[:, keep].sum(1, keepdim=True)
        assert bool(((pk @ v[keep].double() - out).abs() > tol).any()), at
