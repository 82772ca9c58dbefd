"""Attention over the paged 4-bit cache where logits are as large as 32 bits hold, and past that.

Tolerances.  Where one key is far ahead of all others the output is its value: as in test_gpu_kv4.  Log-sum-exp is that key's logit:
D products summed in 32 bits (at most D / 2 = 64 roundings of 2^-24 that add up, 4e-6 of it) and three more roundings.
"""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from test_gpu_kv4 import TYPES, Problem, host, kv4  # noqa: F401  (kv4 is the fixture)

pytestmark = pytest.mark.gpu

# single tokens and drafts of 8 and of 32 rows; chunks with tiles of up to 64 rows and of more; caches of one and of many workgroups
SHAPES = [(8, 2, [700, 33, 3, 2500], [1, 1, 1, 1]), (8, 2, [700, 33, 3], [8, 2, 3]), (4, 1, [90, 700], [12, 9]), (8, 2, [700, 64, 130], [100, 12, 20])]


def extreme(kv4, shape, D, dtype, c, near):  # noqa: F811
    """Keys below zero and queries of the one value c, so that all logits have the sign of -c; of every request's first tokens that
    all its rows see, one key is `near` as far from zero as the others or nearer."""
    H, Hkv, lens, news = shape
    first = np.concatenate([[0], np.cumsum(lens)])
    ahead = [int(first[r] + (lens[r] - news[r]) // 2) for r in range(len(lens))]

    def values(k, v):
        k[:] = -(0.5 + np.abs(k))
        for t in ahead if near != 1 else ():
            k[t] *= near

    p = Problem(kv4, lens, news, H, Hkv, D, 32, TYPES[dtype], values=values, seed=D)
    p.q = torch.full(p.q.shape, c, dtype=TYPES[dtype], device="cuda")
    return p


def check_one_ahead(p):
    out, lse, q = host(p.run()), host(p.lse), host(p.q).astype(np.float64)
    first = np.concatenate([[0], np.cumsum(p.lens)])
    for r, n in enumerate(p.news):
        mine = slice(int(p.start[r]), int(p.start[r + 1]))
        for g in range(p.Hkv):
            heads = slice(g * p.G, (g + 1) * p.G)
            k, v = p.k[first[r]:first[r + 1], g], p.v[first[r]:first[r + 1], g]
            ref, ref_lse, spread = orc.attention(q[mine, heads], k, v, n, p.scale)
            tol = 5e-5 * spread + (np.abs(ref) * 2.0 ** -8 if p.dtype == torch.bfloat16 else 0)
            assert np.all(np.abs(out[mine, heads] - ref) <= tol), (r, g)
            assert np.all(np.abs(lse[mine, heads] - ref_lse) <= 5e-6 * np.abs(ref_lse)), (r, g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
def test_large_logits_of_either_sign(kv4, shape, D, dtype):  # noqa: F811
    for c in (1e7, 1e10, 1e20, 1e31, 1e35):
        check_one_ahead(extreme(kv4, shape, D, dtype, c, 0.25))
        check_one_ahead(extreme(kv4, shape, D, dtype, -c, 4.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_logits_that_overflow_are_infinite(kv4, shape, dtype):  # noqa: F811
    """Rows whose every logit is -infinity are NaN, and so are those with one of +infinity; rows that see nothing stay zeros; a
    key of -infinity among others has no weight."""
    for c in (3e38, -3e38):
        p = extreme(kv4, shape, 128, dtype, c, 1.0)
        assert np.isnan(host(p.run())).all() and np.isnan(host(p.lse)).all()
    check_one_ahead(extreme(kv4, shape, 128, dtype, 3e38, 2.0 ** -60))      # one finite logit
    H, Hkv, lens, news = shape
    short = (H, Hkv, [max(n - 1, 0) for n in news], news)                   # the first token of every request sees nothing
    p = extreme(kv4, short, 128, dtype, 3e38, 1.0)
    out, lse = host(p.run()), host(p.lse)
    for r in range(len(news)):
        a, b = int(p.start[r]), int(p.start[r + 1])
        assert not out[a].any() and np.isneginf(lse[a]).all()
        assert np.isnan(out[a + 1:b]).all() and np.isnan(lse[a + 1:b]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("news", [[1, 1], [6, 2], [20, 16], [60, 50]])
def test_finite_logits_come_before_and_after_infinite_ones(kv4, news, dtype):  # noqa: F811
    """Stretches of -infinity that are longer than any workgroup's share, with the finite logits at one end."""
    lens = [3000, 2600]
    for at_end in (False, True):
        def values(k, v):
            k[:] = -(0.5 + np.abs(k))
            for start, n in ((0, lens[0]), (lens[0], lens[1])):
                near = slice(start + n - 200, start + n - 100) if at_end else slice(start, start + 100)
                k[near] *= 2.0 ** -125      # logits of some -30
        p = Problem(kv4, lens, news, 4, 1, 128, 64, TYPES[dtype], values=values, seed=news[0])
        p.q = torch.full(p.q.shape, 3e38, dtype=TYPES[dtype], device="cuda")
        p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_large_logits_stay_in_their_rows(kv4, shape, dtype):  # noqa: F811
    """Rows of ordinary queries next to rows whose logits are equal and huge: those take the mean of what they see."""
    H, Hkv, lens, news = shape

    def values(k, v):
        k[:, :, 64:] = -1.0
    for c in (2e9, 1e30, -1e30):
        p = Problem(kv4, lens, news, H, Hkv, 128, 32, TYPES[dtype], values=values, seed=len(lens))
        p.q[:, :, 64:] = 0
        large = torch.rand((len(p.q), H), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") < 0.3
        q = torch.zeros_like(p.q)
        q[:, :, 64:] = c
        p.q = torch.where(large[:, :, None], q, p.q)
        out, lse = p.run(), p.lse.clone()
        want = p.scale * 64 * -1.0 * q[0, 0, 64].double()       # of every key
        first, large = np.concatenate([[0], np.cumsum(lens)]), large.cpu().numpy()
        for r, n in enumerate(news):
            for t in range(n):
                for h in np.nonzero(large[p.start[r] + t])[0]:
                    seen = p.v[first[r]:first[r] + lens[r] - n + t + 1, h // p.G]
                    got, mean = host(out)[p.start[r] + t, h], seen.mean(axis=0)
                    assert np.all(np.abs(got - mean) <= 5e-5 * np.abs(seen).mean(axis=0) + (np.abs(mean) * 2.0 ** -8 if dtype == "bf16" else 0))
                    assert abs(float(lse[p.start[r] + t, h]) - float(want)) <= 5e-6 * abs(float(want))
        p.q = torch.where(torch.from_numpy(large).cuda()[:, :, None], torch.zeros_like(p.q), p.q)
        again = p.run()
        keep = ~torch.from_numpy(large).cuda()
        assert torch.equal(again[keep], out[keep]) and torch.equal(p.lse[keep], lse[keep])
        p.check(again)
