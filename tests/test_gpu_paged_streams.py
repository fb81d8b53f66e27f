"""The paged key-value cache on streams other than the one its object was made on: counters and status word are clear before any call, and the
object's own memory is not given out again under a call that is still running."""
import pytest
import torch

import paged_util as U
from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
HEADS = (8, 2, 64)


def _pool():
    return U.Pool([3000, 1200], HEADS, BF, 16)             # long enough that runs cut units: parts are joined


def _object(pool):
    from paper_2603_05454_b200 import PagedKVCache
    return PagedKVCache(pool.k, pool.v, pool.table, n_heads=HEADS[0], weights=True)


def _want(pool, q):
    out = torch.empty_like(q)
    _object(pool).attention(q, pool.lens, out)
    torch.cuda.synchronize()
    return out


def _dirty(n):
    """Memory that the allocator hands out next holds no zeros."""
    for size in (n, 1):
        torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    torch.full((1,), -1, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("how", ["argument", "current"])
def test_a_call_on_another_stream_right_after_the_construction(how):
    pool = _pool()
    q = torch.randn(2, HEADS[0] * 64, device=DEV).to(BF)
    want, out, side = _want(pool, q), torch.zeros_like(q), torch.cuda.Stream()
    _dirty(_object(pool).workspace.numel())
    torch.cuda.synchronize()
    torch.cuda._sleep(400_000_000)                          # the stream of the construction is a fifth of a second behind
    c = _object(pool)
    if how == "argument":
        c.attention(q, pool.lens, out, stream=side)
    else:
        with torch.cuda.stream(side):
            c.attention(q, pool.lens, out)
    side.synchronize()
    got = out.clone()
    torch.cuda.synchronize()
    c.attention(q, pool.lens, out)                          # and the counters are clear behind it
    c.check()
    assert torch.equal(got, want) and torch.equal(out, want)


def test_memory_of_a_dropped_object_waits_for_its_calls():
    pool = _pool()
    q = torch.randn(2, HEADS[0] * 64, device=DEV).to(BF)
    want, out, side = _want(pool, q), torch.zeros_like(q), torch.cuda.Stream()
    c = _object(pool)
    at, status, n = c.workspace.data_ptr(), c.status.data_ptr(), c.workspace.numel()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
    c.attention(q, pool.lens, out, stream=side)
    del c
    taken = [torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV), *(torch.full((1,), -1, dtype=torch.int32, device=DEV) for _ in range(4))]
    assert all(t.data_ptr() not in (at, status) for t in taken)
    side.synchronize()
    assert torch.equal(out, want) and all(bool((t == (255 if t.dtype == torch.uint8 else -1)).all()) for t in taken)


def test_a_status_that_was_raised_is_clear_for_the_next_call_on_any_stream():
    from paper_2603_05454_b200 import LSPError
    pool = _pool()
    q = torch.randn(2, HEADS[0] * 64, device=DEV).to(BF)
    out, side, bad = torch.zeros_like(q), torch.cuda.Stream(), pool.lens + pool.cap
    c = _object(pool)
    word = c.status

    class Late:
        """The status word, cleared on a stream that is a fifth of a second behind."""
        item = word.item

        def zero_(self):
            torch.cuda._sleep(400_000_000)
            word.zero_()

    torch.cuda.synchronize()
    c.attention(q, bad, out)
    c.status = Late()
    with pytest.raises(LSPError):
        c.check()
    c.status = word
    c.attention(q, bad, out, stream=side)
    with pytest.raises(LSPError):
        c.check()
    c.check()


def test_a_stream_from_outside_torch_may_be_gone_before_the_object():
    import ctypes as C
    cuda = C.CDLL("libcudart.so.12")
    handle, pool = C.c_void_p(), _pool()
    q = torch.randn(2, HEADS[0] * 64, device=DEV).to(BF)
    want, out = _want(pool, q), torch.zeros_like(q)
    assert cuda.cudaStreamCreateWithFlags(C.byref(handle), 1) == 0
    c = _object(pool)
    torch.cuda.synchronize()
    c.attention(q, pool.lens, out, stream=torch.cuda.ExternalStream(handle.value))
    assert cuda.cudaStreamSynchronize(handle) == 0 and torch.equal(out, want)
    assert cuda.cudaStreamDestroy(handle) == 0
    n = c.workspace.numel()
    del c
    assert bool((torch.full((n,), 3, dtype=torch.uint8, device=DEV) == 3).all())


def test_the_first_call_in_a_capture_and_the_object_dropped_behind_the_graph():
    pool = _pool()
    q = torch.randn(2, HEADS[0] * 64, device=DEV).to(BF)
    want, out, graph = _want(pool, q), torch.zeros_like(q), torch.cuda.CUDAGraph()
    c = _object(pool)
    at, n = c.workspace.data_ptr(), c.workspace.numel()
    with torch.cuda.graph(graph):
        c.attention(q, pool.lens, out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    out.zero_()
    c.attention(q, pool.lens, out)                          # eagerly, on the stream of the construction
    c.check()
    assert torch.equal(out, want)
    del graph, c
    torch.cuda.synchronize()
    again = [torch.full((n,), 3, dtype=torch.uint8, device=DEV) for _ in range(2)]
    assert all(bool((t == 3).all()) for t in again)


def test_an_object_made_in_a_capture_is_the_graphs_own():
    """Its clears are replayed with the graph, ahead of the calls on every stream of the capture; an eager call is an error, not a wrong result."""
    pool = _pool()
    q = torch.randn(2, HEADS[0] * 64, device=DEV).to(BF)
    want, outs, graph, side = _want(pool, q), [torch.zeros_like(q) for _ in range(2)], torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)                              # forked ahead of the construction
        c = _object(pool)
        c.attention(q, pool.lens, outs[0], stream=side)
        main.wait_stream(side)
        c.attention(q, pool.lens, outs[1])
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    with pytest.raises(RuntimeError):
        c.attention(q, pool.lens, outs[0])
    torch.cuda.synchronize()
    del graph, c
