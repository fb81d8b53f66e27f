"""A call of the paged cache whose launch has more than 2^31 threads."""
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu


def test_append_of_more_blocks_than_31_bits_of_threads():
    """2^23 rows and a few, a block each: all but the first lie behind the sequence's last slot."""
    from paper_2603_05454_b200 import LSPError, PagedKVCache
    heads, n = 33, (1 << 23) + 5
    if torch.cuda.mem_get_info()[0] < 50 << 30:
        pytest.skip("needs 35 GB")
    new = torch.empty(n, heads * 64, dtype=torch.bfloat16, device=DEV)
    new[:64] = torch.randn(64, heads * 64, device=DEV)
    k, v = (torch.zeros(4, 16, heads, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lens, lens_out = (torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2))
    table = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device=DEV)
    c = PagedKVCache(k, v, table, n_heads=heads)
    c.append(new, new, lens, lens_out)
    with pytest.raises(LSPError) as e:
        c.check()
    assert "status 1)" in str(e.value) and lens_out.tolist() == [64]
    for pool in (k, v):
        assert torch.equal(pool[table[0].long()].view(64, -1), new[:64])
    del new
    torch.cuda.empty_cache()
