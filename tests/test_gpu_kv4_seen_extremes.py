"""Windows and trees over the paged 4-bit cache where logits are as large as 32 bits hold and past that, where queries and values are not
finite, and in batches of more requests than a wave and than a workgroup has lanes.

Tolerances.  Outputs: as in test_gpu_kv4_seen.  Log-sum-exp of rows with one key far ahead is that key's logit: D products summed in 32 bits
(at most D / 2 = 64 roundings of 2^-24 that add up, 4e-6 of it) and three more roundings: 5e-6 of it.
"""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from test_gpu_kv4 import TYPES, host, kv4  # noqa: F401  (kv4 is the fixture)
from test_gpu_kv4_seen import Seen

pytestmark = pytest.mark.gpu

# single tokens, drafts of 8 and of 32 rows, of up to 64 rows and of more; caches of one and of many workgroups
SHAPES = [(8, 2, [700, 33, 3, 2500], [1, 1, 1, 1]), (8, 2, [700, 33, 3], [8, 2, 3]), (4, 1, [90, 700], [12, 9]), (8, 2, [700, 64, 130], [100, 12, 20])]
KINDS = [None, "tree", "chain"]


def extreme(kv4, shape, kind, D, dtype, c, near):  # noqa: F811
    """Keys below zero and queries of the one value c, so that all logits have the sign of -c; one key of each request, in the window of all
    its rows, is `near` as far from zero as the others or nearer."""
    H, Hkv, lens, news = shape
    first = np.concatenate([[0], np.cumsum(lens)])
    ahead = [int(first[r] + (lens[r] - news[r]) // 2) for r in range(len(lens))]

    def values(k, v):
        k[:] = -(0.5 + np.abs(k))
        for t in ahead if near != 1 else ():
            k[t] *= near

    p = Seen(kv4, lens, news, H, Hkv, D, 32, TYPES[dtype], values=values, seed=D)
    p.set(max(-(-(n - m) // 2) + m + 1 for n, m in zip(lens, news)), 2, kind)
    p.q = torch.full(p.q.shape, c, dtype=TYPES[dtype], device="cuda")
    p.ahead = [t - int(first[r]) for r, t in enumerate(ahead)]
    return p


def check_one_ahead(p, others_infinite=False):
    """others_infinite: the logits of all other keys are -infinity in 32 bits, so rows that see some of those but not the one are NaN
    (where nothing is cached before a tree, the one is its first draft, and not every branch has it)."""
    out, lse, q = host(p.run()), host(p.lse), host(p.q).astype(np.float64)
    first = np.concatenate([[0], np.cumsum(p.lens)])
    for r in range(len(p.news)):
        mine, seen = np.arange(int(p.start[r]), int(p.start[r + 1])), p.seen(r)
        if others_infinite:
            lost = seen.any(axis=1) & ~seen[:, p.ahead[r]]
            assert np.isnan(out[mine[lost]]).all() and np.isnan(lse[mine[lost]]).all()
            mine, seen = mine[~lost], seen[~lost]
        for g in range(p.Hkv):
            heads = slice(g * p.G, (g + 1) * p.G)
            k, v = p.k[first[r]:first[r + 1], g], p.v[first[r]:first[r + 1], g]
            ref, ref_lse, spread = orc.seen_attention(q[mine, heads], k, v, seen, p.scale)
            tol = 5e-5 * spread + (np.abs(ref) * 2.0 ** -8 if p.dtype == torch.bfloat16 else 0)
            assert np.all(np.abs(out[mine, heads] - ref) <= tol), (r, g)
            np.testing.assert_array_equal(np.isneginf(lse[mine, heads]), np.isneginf(ref_lse))
            there = np.isfinite(ref_lse)
            assert np.all(np.abs(lse[mine, heads] - ref_lse)[there] <= 5e-6 * np.abs(ref_lse)[there]), (r, g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_large_logits_of_either_sign(kv4, shape, kind, D, dtype):  # noqa: F811
    for c in (1e7, 1e20, 1e35):
        check_one_ahead(extreme(kv4, shape, kind, D, dtype, c, 0.25))
        check_one_ahead(extreme(kv4, shape, kind, D, dtype, -c, 4.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_logits_that_overflow_are_infinite(kv4, shape, kind, dtype):  # noqa: F811
    """Rows whose every logit is -infinity are NaN, and so are those with one of +infinity; a key of -infinity among others has no weight."""
    for c in (3e38, -3e38):
        p = extreme(kv4, shape, kind, 128, dtype, c, 1.0)
        out, lse = host(p.run()), host(p.lse)
        for r, n in enumerate(p.news):
            sees = p.seen(r).any(axis=1)
            mine = slice(int(p.start[r]), int(p.start[r]) + n)
            assert np.isnan(out[mine][sees]).all() and np.isnan(lse[mine][sees]).all()
            assert not out[mine][~sees].any() and np.isneginf(lse[mine][~sees]).all()
    check_one_ahead(extreme(kv4, shape, kind, 128, dtype, 3e38, 2.0 ** -60), True)      # one finite logit


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("news", [[1, 1], [6, 2], [20, 16], [60, 50]])
@pytest.mark.parametrize("kind,window", [(None, 2000), ("any", 0), ("tree", 2000)])
def test_finite_logits_come_before_and_after_infinite_ones(kv4, kind, window, news, dtype):  # noqa: F811
    """Stretches of -infinity that are longer than any workgroup's share, with the finite logits at one end of what is seen."""
    lens = [3000, 2600]
    for at_end in (False, True):
        def values(k, v):
            k[:] = -(0.5 + np.abs(k))
            for start, n in ((0, lens[0]), (lens[0], lens[1])):
                near = slice(start + n - 200, start + n - 100) if at_end else slice(start, start + 100)
                k[near] *= 2.0 ** -125      # logits of some -30
        p = Seen(kv4, lens, news, 4, 1, 128, 64, TYPES[dtype], values=values, seed=news[0]).set(window, 90, kind)
        p.q = torch.full(p.q.shape, 3e38, dtype=TYPES[dtype], device="cuda")
        p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("news", [1, 3, 8, 12, 40, 100])
@pytest.mark.parametrize("kind", [None, "any"])
def test_values_without_weight(kv4, kind, news, D, dtype):  # noqa: F811
    """All weight is on one key that every row sees (logits apart by more than 150): a value that is not finite makes its group of
    channels NaN in the rows that see it, and in no other."""
    length, window = 700, 400
    ends = length - news
    ahead = ends - 5
    for bad in (1, 100, ends - window - 3, ends - window + news // 2 + 1, ends - 40, ends - 6, ends - 4, ends, ends + news // 2, length - 1):
        def values(k, v):
            k[ahead], v[bad, :, 40:] = 6.0, np.inf
        p = Seen(kv4, [length], [news], 4, 1, D, 32, TYPES[dtype], values=values, seed=news).set(window, 4, kind)
        p.q.fill_(4.0)
        out, lse = host(p.run()), host(p.lse)
        sees = p.seen(0)[:, bad]
        assert np.isfinite(lse).all(), bad
        assert np.isfinite(out[:, :, :32]).all() and np.isfinite(out[~sees]).all(), bad
        assert np.isnan(out[sees][:, :, 32:]).all(), bad
        np.testing.assert_array_equal(out[:, :, :32], np.broadcast_to(p.v[ahead, 0, :32].astype(np.float32), out[:, :, :32].shape))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("news", [[2, 1], [8, 5], [14, 16], [50, 40]])
def test_queries_that_are_not_finite_stay_in_their_rows(kv4, news, kind, dtype):  # noqa: F811
    p = Seen(kv4, [900, 60], news, 8, 2, 128, 64, TYPES[dtype]).set(100, 3, kind)
    want = p.run().clone()
    lse = p.lse.clone()
    last = sum(news) - 1
    p.q[1, 3], p.q[last, 0, 5] = float("nan"), float("inf")
    out = p.run()
    for at in ((1, 3), (last, 0)):
        assert torch.isnan(out[at]).all() and torch.isnan(p.lse[at])
        out[at], p.lse[at] = want[at], lse[at]
    assert torch.equal(out, want) and torch.equal(p.lse, lse)


@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.bfloat16), (64, torch.float32)])
@pytest.mark.parametrize("requests", [70, 300])
@pytest.mark.parametrize("kind,window", [(None, 25), ("tree", 0), ("any", 25)])
def test_drafts_and_chunks_of_many_requests(kv4, kind, window, requests, D, dtype):  # noqa: F811
    rng = np.random.default_rng(requests)
    news = rng.integers(0, 40, requests)
    news[::3] = 1
    lens = news + rng.integers(0, 60, requests)
    p = Seen(kv4, lens.tolist(), news.tolist(), 8, 2, D, 32, dtype, seed=requests).set(window, 2, kind)
    p.check(p.run())
    few = np.minimum(news, 4)
    p = Seen(kv4, lens.tolist(), few.tolist(), 8, 2, D, 32, dtype, seed=requests).set(window, 2, kind)
    p.check(p.run())
