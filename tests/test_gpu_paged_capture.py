"""PagedCache under graph capture: refused, and neither the capture nor the cache is the worse for it."""
import pytest
import torch

from paper_2408_10188_amd import paged
from tests.helpers import DEV, nans_like

pytestmark = pytest.mark.gpu


def test_paged_cache_calls_in_a_capture_raise():
    cache = paged.PagedCache(1, 8, 16, 4, 2, 128, 64, torch.bfloat16, DEV)
    a = cache.add()
    cache.step([a], [5])
    q, k, v = (torch.randn(5, h, 128, device=DEV).bfloat16() for h in (4, 2, 2))
    x, y = torch.arange(8.0, device=DEV), torch.zeros(8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: cache.step([a], [1]), cache.compact, lambda: cache.append(0, None, None, q, k, v), lambda: cache.attend(0, q)):
            with pytest.raises(RuntimeError, match="captured"):
                call()
        y.copy_(x * 2)
    for i in range(3):
        x += 1
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, x * 2)
    before = q.clone()
    assert cache.append(0, None, None, q, k, v) is q and torch.equal(q, before)
    o = nans_like(q)
    assert cache.attend(0, q, o_final=o) is o and bool(torch.isfinite(o).all())
    assert torch.equal(o[0], v[0].repeat_interleave(2, 0))      # the first token sees itself alone
    assert cache.lengths == {a: 5}
