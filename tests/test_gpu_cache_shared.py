"""Pages that several table entries name are not written by append: the tokens are left out and reported."""
import numpy as np
import pytest
import torch

from paper_2607_09385_b200 import binding as B

from test_gpu_cache import contents, expected_values, ints, make_cache, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,seq", [(2, 1), (2, 5), (2, 40), (100, 40), (300, 40)])  # a warp a token; the last a warp a unit
def test_append_leaves_shared_pages_alone(d, heads, seq):
    page, bad = 32, B.STEEL_ERR_INVALID_ARG
    c = make_cache(2, 40, page, heads, d, 4, 8)
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = normal(g, 2, heads, 50, d), normal(g, 2, heads, 50, d)
    c.extend(ints([50, 50]), ints([0, 1]))
    c.append(1, k, v, slots=ints([0, 1]))
    # slot 2 takes over slot 0's pages: until one of the two is extended neither's tokens may be written
    c.fork(ints([0]), ints([2]))
    assert c.last_status() == B.STEEL_OK
    pool = c.pool.clone()
    x, y = normal(g, 1, heads, seq, d), normal(g, 1, heads, seq, d)
    for slot in (0, 2):
        c.append(1, x, y, slots=ints([slot]))
        assert c.last_status() == bad and torch.equal(c.pool, pool)
    # no tokens: nothing to report
    c.append(1, x, y, ints([0]), ints([2]))
    assert c.last_status() == B.STEEL_OK and torch.equal(c.pool, pool)
    # the other sequence of a batch is written
    c.append(1, torch.cat((x, x)), torch.cat((y, y)), slots=ints([2, 1]))
    assert c.last_status() == bad
    for got, old, new in zip(contents(c, 1, 1), (k, v), (x, y)):
        assert np.array_equal(got, np.concatenate((expected_values(old[1])[:, :50 - seq], expected_values(new[0])), 1))
    for s in (0, 2):
        for got, old in zip(contents(c, 1, s), (k, v)):
            assert np.array_equal(got, expected_values(old[0]))
    # extended, the child has a last page of its own, and the parent keeps what it had
    c.extend(ints([seq]), ints([2]))
    c.append(1, x, y, slots=ints([2]))
    assert c.last_status() == B.STEEL_OK
    for got, old, new in zip(contents(c, 1, 2), (k, v), (x, y)):
        assert np.array_equal(got, np.concatenate((expected_values(old[0]), expected_values(new[0])), 1))
    for got, old in zip(contents(c, 1, 0), (k, v)):
        assert np.array_equal(got, expected_values(old[0]))
    # more tokens than the child's own pages hold: those on the shared first page are left out
    own = 50 + seq - page
    z = normal(g, 1, heads, own + 3, d)
    c.append(1, z, z, slots=ints([2]))
    assert c.last_status() == bad
    for got, old in zip(contents(c, 1, 2), (k, v)):
        assert np.array_equal(got, np.concatenate((expected_values(old[0])[:, :page], expected_values(z[0])[:, 3:]), 1))
    for got, old in zip(contents(c, 1, 0), (k, v)):
        assert np.array_equal(got, expected_values(old[0]))
    c.close()
