"""The cache's attention where a warp's share is long: look-ups behind the first sixteen steps, rings that go round, several whole segments a
warp, references renewed late, parts of many steps.  Little memory: entries of a batch name the same few slots, whose pages lie in a random
order.  Values and scores have a mean that moves along the sequence, so that a part that is missing, doubled or taken from elsewhere shows."""
import numpy as np
import pytest
import torch

from paper_2607_09385_b200 import binding as B
from paper_2607_09385_b200 import cache as C

import cache_reference as R
from test_gpu_cache import contents, ints, make_cache, normal, state

pytestmark = pytest.mark.gpu
CAUSAL, WINDOW = B.STEEL_MASK_CAUSAL, B.STEEL_MASK_WINDOW


def scattered(lens, d, page, heads, seed):
    """Slot s holds lens[s] tokens, on pages in a random order.  Values drift by a standard deviation over 300 tokens."""
    held = [-(-n // page) for n in lens]
    pages = sum(held) + 3
    c = make_cache(1, pages, page, heads, d, len(lens), max(held) + 1)
    g = torch.Generator(device="cuda").manual_seed(seed)
    c.extend(ints(lens))
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    c.table.copy_(torch.where(c.table >= 0, order[c.table.clamp(min=0).long()], c.table))
    c.refs.zero_()
    c.refs[c.table[c.table >= 0].long()] = 1
    for s, n in enumerate(lens):
        if n:
            drift = torch.arange(n, device="cuda").float()[:, None] / 300
            k = normal(g, 1, heads, n, d)
            v = (normal(g, 1, heads, n, d).float() + torch.sin(drift + torch.arange(d, device="cuda")) * 2).to(torch.bfloat16)
            c.append(0, k, v, slots=ints([s]))
    assert c.last_status() == B.STEEL_OK
    return c, g


def share_of(c, slots, lens, counts, group, seq_q, flags, window):
    """Units of work a warp gets: 32 tokens each and two a segment (sequence, head, 8 rows)."""
    heads, tiles = c.heads_kv, -(-group * seq_q // 8)
    total = 0
    for s, n in zip(slots, counts):
        first = max(0, lens[s] - n - window + 1) // 32 if flags & WINDOW else 0
        total += (max(1, -(-lens[s] // 32) - first) + 2) * heads * tiles if n else 0
    return -(-total // (torch.cuda.get_device_properties(0).multi_processor_count * 16))


def compare(c, g, slots, group, seq_q, counts, flags, window, scale):
    """Against 64 bits.  Bounds, element by element: 2^-8 of the result; the fp16 rounding of weights times scales (2^-11) and the scores' ((head_dim + 16) of
    2^-23 of `size`, tests/cache_reference.py), which are independent from token to token and uniform: seven standard deviations of their sum, code times
    scale and zero by themselves; sums of 512 tokens cut off one way, 2^-18 of them, and the joined sum by 2^-23 of it for each 16 tokens."""
    n, heads, d = len(slots), c.heads_kv, c.head_dim
    q = normal(g, n, heads * group, seq_q, d)
    o = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    c.attend(0, q, scale, ints(counts), ints(slots), flags, window, o, lse)
    assert c.last_status() == B.STEEL_OK
    again = torch.full_like(q, 7.0)
    c.attend(0, q, scale, ints(counts), ints(slots), flags, window, again)
    for i in range(n):
        m = counts[i]
        assert (o[i, :, m:] == 7).all() and (lse[i, :, m:] == 7).all()
    assert torch.equal(o, again)
    cached = {}
    for i, s in enumerate(slots):
        m = counts[i]
        if m == 0:
            continue
        if s not in cached:
            kk, vv = (torch.from_numpy(x).cuda() for x in contents(c, 0, s))  # [heads, tokens, channels]
            x = vv.reshape(*vv.shape[:2], d // 64, 64)
            low = x.min(-1, keepdim=True)[0]
            cached[s] = kk, vv, (x - low + low.abs()).reshape(vv.shape)
        kk, vv, mass = cached[s]
        tokens = kk.shape[1]
        qq = q[i, :, :m].double().reshape(heads, group * m, d)
        pos = (tokens - m + torch.arange(m, device="cuda")).repeat(group)[:, None]
        j = torch.arange(tokens, device="cuda")[None]
        seen = torch.ones((group * m, tokens), dtype=torch.bool, device="cuda")
        if flags & CAUSAL:
            seen &= j <= pos
        if flags & WINDOW:
            seen &= pos - j < window
        score = (qq @ kk.transpose(1, 2) * scale).masked_fill(~seen, -torch.inf)
        want_l = torch.logsumexp(score, -1)
        none = torch.isneginf(want_l)
        p = torch.exp(score - want_l.masked_fill(none, 0)[..., None])
        ref = p @ vv
        size = scale * qq.abs().sum(-1, keepdim=True) * 2 * kk.abs().amax((1, 2), keepdim=True) if tokens else torch.zeros_like(ref[..., :1])
        rel = 2.0 ** -11 + (d + 17) * 2.0 ** -23 * size + 2.0 ** -21
        total = p @ mass
        tol = 2.0 ** -8 * ref.abs() + 7 * rel / 3 ** 0.5 * ((p * p) @ (mass * mass)).sqrt() + 2.0 ** -18 * total + \
            2.0 ** -23 * (tokens / 16 + 32) * 3 * ref.abs().amax(-1, keepdim=True)
        got = o[i, :, :m].double().reshape(ref.shape)
        assert ((got - ref).abs() <= tol).all(), (i, s, float(((got - ref).abs() / tol.clamp(min=1e-30)).max()))
        got_l = lse[i, :, :m].double().reshape(want_l.shape)
        assert torch.equal(torch.isneginf(got_l), none)
        assert ((got_l - want_l).abs()[~none] <= (rel[..., 0] + 2.0 ** -22 * (1 + want_l.abs()) + 2.0 ** -24 * (tokens / 8 + 32))[~none]).all()


CASES = [
    # lens, batch, heads, group, seq_q, ragged counts, flags, window, least share
    ([2000, 1999, 31], 64, 8, 8, 1, False, CAUSAL, 0, 10),          # a part of a segment in each warp
    ([2000, 513, 1, 0, 1024], 200, 4, 4, 6, True, CAUSAL, 0, 17),   # ragged, rows behind the last query
    ([40, 70, 0, 100, 33], 300, 8, 2, 9, True, CAUSAL, 0, 10),      # several whole segments a warp
    ([9000], 60, 2, 16, 5, False, CAUSAL, 0, 100),                  # whole segments and more: look-ups behind the sixteenth step
    ([5000, 4097], 80, 4, 4, 10, True, CAUSAL | WINDOW, 1500, 20),  # windows that begin within a step
    ([3000, 2049], 70, 4, 5, 7, True, WINDOW, 700, 12),
    ([7777], 60, 4, 8, 3, False, 0, 0, 40),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_long_shares(d, case):
    lens, batch, heads, group, seq_q, ragged, flags, window, least = CASES[case]
    c, g = scattered(lens, d, [16, 32, 64, 128][(case + d // 64) % 4], heads, 10 + case)
    rng = np.random.default_rng(case)
    slots = [int(s) for s in rng.integers(0, len(lens), batch)]
    counts = [int(x) for x in rng.integers(0, seq_q + 1, batch)] if ragged else [seq_q] * batch
    assert share_of(c, slots, lens, counts, group, seq_q, flags, window) >= least
    compare(c, g, slots, group, seq_q, counts, flags, window, 0.3 * d ** -0.5)
    c.close()


@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_rise_along_a_long_share(d):
    # the reference is renewed again and again, in steps far behind a warp's first
    tokens, heads, batch, rows = 6000, 2, 60, 160
    c = make_cache(1, 200, 32, heads, d, 1, 200)
    g = torch.Generator(device="cuda").manual_seed(31)
    c.extend(ints([tokens]))
    q1 = normal(g, 1, 1, 1, d)
    direction = q1[0, 0, 0].float() / float(q1.float().square().sum())
    ramp = torch.arange(tokens, device="cuda").float()[:, None] / 200 * d ** 0.5   # 30 in all
    k = (normal(g, 1, heads, tokens, d, scale=0.3).float() + direction * ramp).to(torch.bfloat16)
    v = normal(g, 1, heads, tokens, d)
    c.append(0, k, v)
    q = q1.expand(batch, heads, rows, d).contiguous()
    q[:, :, 1::2] = -q[:, :, 1::2]  # every other row sees them fall
    scale = d ** -0.5
    assert share_of(c, [0] * batch, [tokens], [rows] * batch, 1, rows, 0, 0) >= 100
    o, lse = c.attend(0, q, scale, slots=ints([0] * batch), flags=0)
    assert c.last_status() == B.STEEL_OK
    kk, vv = contents(c, 0, 0)
    for h in range(heads):
        for i in (0, 1):
            ref, ref_l, tol, tol_l = R.attend(q[0, h:h + 1, i:i + 1].double().cpu().numpy(), kk[h:h + 1], vv[h:h + 1], scale, 0, 0)
            got = o[:, h, i::2].double().cpu().numpy()
            assert (np.abs(got - ref[0]) <= tol[0]).all() and (np.abs(lse[:, h, i::2].double().cpu().numpy() - ref_l[0]) <= tol_l[0]).all()
            assert np.abs(ref).max() > 2 * tol.max()  # what a few hundred tokens weigh
    c.close()


def test_pages_meet_every_outcome():
    # random calls on a small pool: each outcome comes about many times, and the cache is the model's after each
    rng = np.random.default_rng(11)
    page, slots, pages, max_pages = 16, 9, 24, 6
    c = make_cache(1, pages, page, 1, 64, slots, max_pages)
    m = R.Model(pages, page, slots, max_pages)
    seen = {}
    for _ in range(400):
        op = str(rng.choice(["extend", "extend", "fork", "free"]))
        n = int(rng.integers(1, 4))
        some = [int(s) for s in rng.permutation(slots)[:n]]
        if rng.random() < 0.1:
            some[0] = int(rng.choice([-1, slots]))
        if op == "extend":
            counts = [int(x) for x in rng.choice([0, 1, 16, 40, -1], n, p=[.1, .3, .3, .25, .05])]
            want = m.extend(some, counts)
            c.extend(ints(counts), ints(some))
        elif op == "fork":
            src = [int(s) for s in rng.integers(0, slots, n)]
            want = m.fork(src, some)
            c.fork(ints(src), ints(some))
        else:
            keep = [int(rng.integers(0, m.lens[s] + 2)) if 0 <= s < slots else 0 for s in some]
            want = m.free(some, keep)
            c.free(ints(some), ints(keep))
        seen[op, want] = seen.get((op, want), 0) + 1
        assert c.last_status() == {"ok": B.STEEL_OK, "invalid": B.STEEL_ERR_INVALID_ARG, "no pages": C.STEEL_ERR_NO_PAGES}[want], (op, want)
        table, lens, refs = state(c)
        assert lens == m.lens and refs == m.refs and np.array_equal(table, m.table()), (op, want)
    outcomes = [("extend", "ok"), ("extend", "invalid"), ("extend", "no pages"), ("fork", "ok"), ("fork", "invalid"), ("free", "ok"), ("free", "invalid")]
    assert set(seen) == set(outcomes) and all(seen[x] >= 5 for x in outcomes), seen
    c.close()
