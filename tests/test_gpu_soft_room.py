"""ps_soft's reserved workspace on the device at sizes where the rows of one launch are limited: captured calls cannot grow it."""
import contextlib
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def soft():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1410_8043_amd import ps_soft

    return ps_soft


@contextlib.contextmanager
def capture(graph):
    """torch.cuda.graph without the garbage collector, which may not free another graph inside a capture."""
    gc.collect()
    gc.disable()
    try:
        with torch.cuda.graph(graph):
            yield
    finally:
        gc.enable()


@pytest.mark.parametrize("n,M,K,dtype,k", [(62_884, 95_190, 34, torch.float16, 1), (40_000, 100_000, 32, torch.float32, 4)])
def test_search_without_exclusions_of_more_rows_than_a_launch(soft, n, M, K, dtype, k):
    g = torch.Generator().manual_seed(K)
    X, W = torch.randn(n, K, generator=g).to(dtype).cuda(), torch.randn(M, K, generator=g).to(dtype).cuda()
    ptr = torch.arange(0, 2 * n + 1, 2).cuda()
    item = torch.randint(0, M, (2 * n,), generator=g, dtype=torch.int32).cuda()
    with soft.PsSoft(M, K, dtype) as h, soft.PsSoft(M, K, dtype) as eager:
        h.reserve(n, 2 * n, k)
        want = eager.top(X, W, k), eager.top(X, W, k, row_ptr=ptr, item=item)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with capture(graph):
            got = h.top(X, W, k), h.top(X, W, k, row_ptr=ptr, item=item)
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        del graph
