"""Sums of the cache's attention over long chains in one warp, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2607_09385_b200 import binding as B

from test_gpu_cache import contents, ints, make_cache, normal

pytestmark = pytest.mark.gpu


def long_cache(d, tokens, heads, page=128, seed=0):
    """One sequence on pages in a random order."""
    pages = -(-tokens // page) + 5
    c = make_cache(1, pages, page, heads, d, 1, pages)
    c.extend(ints([tokens]))
    held = -(-tokens // page)
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = torch.randperm(pages, generator=g, device="cuda")[:held].to(torch.int32)
    c.table[0, :held] = order
    c.refs.zero_()
    c.refs[order.long()] = 1
    return c, g


def parts_of(v):
    """Values float64 [tokens, channels] -> code times scale, magnitude of zero, scale (bounds, by group): code 0 stands for the least."""
    n = v.shape[1] // 64
    x = v.reshape(v.shape[0], n, 64)
    low = x.min(-1, keepdims=True)
    wide = lambda a: np.broadcast_to(a, x.shape).reshape(v.shape)  # noqa: E731
    return (x - low).reshape(v.shape), wide(np.abs(low)), wide((x.max(-1, keepdims=True) - low) / 15)


@pytest.mark.parametrize("d,tokens", [(64, 16384), (128, 16384), (64, 65536), (128, 32768)])
def test_long_chains_in_one_warp(d, tokens):
    """As many rows as give each warp a whole sequence's steps, one after the other: the codes' sums grow with the chain while their zeros
    take them back, and the mean of the values shrinks.

    RMS bounds.  The result's rounding is uniform within 2^-8 of it: 2^-8 / sqrt(3).  A weight times its scale is rounded to fp16, independently
    of the others, uniform within 2^-11, and a score's roundings ((head_dim + 16) of 2^-23 of `size`, tests/cache_reference.py) are as independent:
    the root of the sum of squares over the tokens, with code times scale and zero as they are summed.  The matrix products' sums may be cut off
    one way by 2^-23 each: 32 products in a row (16 steps, 512 tokens) before zeros join them, on average half of what the 512 tokens add up to, 2^-19 of
    all codes' sum; and 2^-23 of the joined sum, which is no larger than a few times the result, for each product of the chain."""
    heads, batch = 2, 64
    warps = torch.cuda.get_device_properties(0).multi_processor_count * 16
    rows = -(-warps // (batch * heads)) * 8
    c, g = long_cache(d, tokens, heads)
    k, v = normal(g, 1, heads, tokens, d), normal(g, 1, heads, tokens, d)
    c.append(0, k, v)
    q = normal(g, batch, heads, rows, d)
    scale = 0.1 / d ** 0.5
    o, lse = c.attend(0, q, scale, slots=ints([0] * batch), flags=0)
    assert c.last_status() == B.STEEL_OK
    kc, vc = contents(c, 0, 0)
    for h in range(heads):
        kk, vv = (torch.from_numpy(x[h]).cuda() for x in (kc, vc))
        su, z, _ = (torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in parts_of(vc[h]))
        for b in (0, 31, 63):
            qq = q[b, h].double()
            s = qq @ kk.T * scale
            p = torch.softmax(s, -1)
            ref = p @ vv
            size = float(scale * qq.abs().sum(-1).max() * 2 * kk.abs().max())
            rel = 2.0 ** -11 + (d + 16) * 2.0 ** -23 * size + 2.0 ** -21
            square = (2.0 ** -8 * ref) ** 2 / 3 + rel ** 2 / 3 * (p ** 2) @ (su + z) ** 2
            cut = 2.0 ** -19 * (p @ su) + 2.0 ** -23 * (tokens / 16) * 3 * ref.abs()
            tol = 1.05 * float(square.mean().sqrt()) + float((cut ** 2).mean().sqrt())
            got = float((o[b, h].double() - ref).square().mean().sqrt())
            assert got <= tol, (d, tokens, h, b, got, tol, float(ref.square().mean().sqrt()))
            want = torch.logsumexp(s, -1)
            # the sum of the weights in 32 bits: a lane adds an eighth of the tokens one after the other
            assert ((lse[b, h].double() - want).abs() <= rel + 2.0 ** -24 * tokens / 8 + 2.0 ** -22 * (1 + want.abs())).all()
    c.close()
