"""Sums of the cache's attention: long chains in one warp, and quiet values beside loud ones that a row does not see or hardly weighs.
Each against 64 bits, within bounds that count what a row sees with the weight that it has."""
import numpy as np
import pytest
import torch

from paper_2607_09385_b200 import binding as B

from test_gpu_cache import contents, ints, make_cache, normal

pytestmark = pytest.mark.gpu
CAUSAL, WINDOW = B.STEEL_MASK_CAUSAL, B.STEEL_MASK_WINDOW


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


def reference(q, k, v, scale, seen):
    """One row in 64 bits, and how far its channels may be off: 2^-8 of the result; a weight's error (scores, ex2) twice, times the values by
    their weights; 2^-11 of each code times scale; what fp16 cannot hold of weight times scale, 2^-30 of the row's largest at most, times codes of
    15; 32-bit sums of codes and zeros, 2^-17 of theirs."""
    d = q.shape[0]
    k, v = k[seen], v[seen]
    s = scale * (k @ q)
    p = np.exp(s - s.max())
    p /= p.sum()
    o = p @ v
    su, z, step = parts_of(v)
    heavy = p > 1e-30
    size = scale * np.abs(q).sum() * 2 * np.abs(k[heavy]).max()
    weight = (d + 17) * 2.0 ** -23 * size + 2.0 ** -21
    tiny = 15 * 2.0 ** -30 * len(p) * (p[:, None] * step).max(0)
    return o, 2.0 ** -8 * np.abs(o) + 2 * weight * (p @ np.abs(v)) + 2.0 ** -11 * (p @ su) + tiny + 2.0 ** -17 * (p @ (su + z))


def check_rows(c, q, scale, flags, window=0):
    o, lse = c.attend(0, q, scale, flags=flags, window=window)
    assert c.last_status() == B.STEEL_OK
    kk, vv = contents(c, 0, 0)
    n, tokens, group = q.shape[2], kk.shape[1], q.shape[1] // kk.shape[0]
    j = np.arange(tokens)
    for h in range(q.shape[1]):
        for i in range(n):
            pos = tokens - n + i
            seen = np.ones(tokens, bool)
            if flags & CAUSAL:
                seen &= j <= pos
            if flags & WINDOW:
                seen &= pos - j < window
            ref, tol = reference(q[0, h, i].double().cpu().numpy(), kk[h // group], vv[h // group], scale, seen)
            got = o[0, h, i].double().cpu().numpy()
            assert (np.abs(got - ref) <= tol).all(), (h, i, np.abs(got - ref).max(), tol.max(), np.abs(ref).max())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("quiet", [1.0, 1e-2, 1e-3, 1e-4])
@pytest.mark.parametrize("flags,window,at", [(CAUSAL, 0, -1), (CAUSAL, 0, -5), (CAUSAL | WINDOW, 100, -107), (CAUSAL | WINDOW, 100, -103)])
def test_loud_values_that_a_row_does_not_see(d, quiet, flags, window, at):
    # an infinite value (65504 in the cache) in a token that some rows of a tile see and others do not: a draft's last tokens, and one that leaves
    # the window
    n = 512
    c = make_cache(1, 40, 16, 1, d, 1, 40)
    g = torch.Generator(device="cuda").manual_seed(21)
    k, v = normal(g, 1, 1, n, d), normal(g, 1, 1, n, d, scale=quiet)
    v[0, 0, at, 5] = float("inf")
    v[0, 0, at, 6] = -float("inf")
    c.extend(ints([n]))
    c.append(0, k, v)
    check_rows(c, normal(g, 1, 2, 8, d), d ** -0.5, flags, window)
    c.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("quiet", [1.0, 1e-2, 1e-4])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_loud_values_that_hardly_count(d, quiet, where):
    # a token whose score is 60 below the others' and whose values are 65504: its part of the result is 1e-21.  Where it comes first it is the
    # largest until the others come
    n = 500
    c = make_cache(1, 40, 16, 1, d, 1, 40)
    g = torch.Generator(device="cuda").manual_seed(22)
    k, v = normal(g, 1, 1, n, d, scale=0.1), normal(g, 1, 1, n, d, scale=quiet)
    q = normal(g, 1, 1, 1, d).expand(1, 3, 1, d).contiguous()
    # a whole unit in front where it comes first: the step before the others'
    at = {"first": slice(0, 32), "middle": slice(250, 251), "last": slice(n - 1, n)}[where]
    v[0, 0, at, ::2], v[0, 0, at, 1::2] = 65504.0, -65504.0
    direction = q[0, 0, 0].float() / float(q[0, 0, 0].float().square().sum())
    k[0, 0, at] = (-direction * 60 * d ** 0.5).to(torch.bfloat16)
    c.extend(ints([n]))
    c.append(0, k, v)
    check_rows(c, q, d ** -0.5, 0)
    c.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rise", [0.3, 3.0, 25.0])
def test_values_that_fall_while_scores_rise(d, rise):
    # every 40 tokens the scores are `rise` higher and the values 2^-2 of those before, from 2^12 down
    n = 480
    c = make_cache(1, 40, 16, 1, d, 1, 40)
    g = torch.Generator(device="cuda").manual_seed(23)
    block = (torch.arange(n, device="cuda") // 40).float()
    q = normal(g, 1, 1, 1, d).expand(1, 9, 1, d).contiguous()
    direction = q[0, 0, 0].float() / float(q[0, 0, 0].float().square().sum())
    k = (normal(g, 1, 1, n, d, scale=0.1).float() + direction * (block * rise * d ** 0.5)[:, None]).to(torch.bfloat16)
    v = (normal(g, 1, 1, n, d).float() * torch.exp2(12 - 2 * block)[:, None]).to(torch.bfloat16)
    c.extend(ints([n]))
    c.append(0, k, v)
    check_rows(c, q, d ** -0.5, 0)
    c.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size,scale", [(2.0 ** 115, 2.0 ** -118), (2.0 ** 119, 2.0 ** -123), (2.0 ** 125, 2.0 ** -126), (2.0 ** -120, 2.0 ** 120)])
def test_queries_at_the_ends_of_bf16(d, size, scale):
    # scores of ordinary size whatever the queries': the largest numbers of bf16 and small ones
    n = 200
    c = make_cache(1, 20, 16, 1, d, 1, 20)
    g = torch.Generator(device="cuda").manual_seed(24)
    k, v = normal(g, 1, 1, n, d), normal(g, 1, 1, n, d)
    c.extend(ints([n]))
    c.append(0, k, v)
    q = (normal(g, 1, 2, 3, d).float().clamp(-3, 3) / 4 * 2 * size).to(torch.bfloat16)
    assert torch.isfinite(q).all()
    check_rows(c, q, scale, CAUSAL)
    c.close()
