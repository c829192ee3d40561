"""An expired wait of the cache's attention: a CTA that joins the parts of a long sequence gives up at its first look, the kernel returns,
STEEL_ERR_TIMEOUT is reported, and neither later calls nor replays of the same captured launch take what came too late."""
import pytest
import torch

from paper_2607_09385_b200 import binding as B
from paper_2607_09385_b200 import cache as C

from test_gpu_cache import ints, make_cache, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_expired_join_is_reported_and_leaves_nothing_behind(d):
    tokens, page = 20000, 64
    c = make_cache(1, 320, page, 2, d, 1, 320)
    g = torch.Generator(device="cuda").manual_seed(1)
    c.extend(ints([tokens]))
    c.append(0, normal(g, 1, 2, tokens, d), normal(g, 1, 2, tokens, d))
    queries = [normal(g, 1, 8, 1, d) for _ in range(40)]
    want = [c.attend(0, q, 0.1) for q in queries]
    q = queries[0].clone()
    assert c.last_status() == B.STEEL_OK
    C.steel_cache_debug_wait(c.handle, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        o, lse = c.attend(0, q, 0.1)
    expired = 0
    for x, (want_o, want_lse) in zip(queries, want):
        q.copy_(x)
        graph.replay()
        status = c.last_status()
        assert status in (B.STEEL_OK, B.STEEL_ERR_TIMEOUT)
        if status == B.STEEL_OK:  # every part was there at the first look
            assert torch.equal(o, want_o) and torch.equal(lse, want_lse)
        else:
            expired += 1
            assert c.last_status() == B.STEEL_OK  # cleared by the read
    assert expired > 0
    # calls beside the graph, with the default bound
    C.steel_cache_debug_wait(c.handle, -1)
    for x, (want_o, want_lse) in zip(queries, want):
        o, lse = c.attend(0, x, 0.1)
        assert torch.equal(o, want_o) and torch.equal(lse, want_lse)
    assert c.last_status() == B.STEEL_OK
    c.close()
