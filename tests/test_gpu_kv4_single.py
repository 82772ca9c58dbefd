"""Single precision in the paged 4-bit cache's attention: bounds that queries or weights of two bf16 numbers instead of three would
miss.

Inputs are chosen for how little else is rounded: a query has one channel that is not zero, so a logit is the sum of three
products, and rows see few keys.  With u = 2^-24: a logit z is off by 3 u |z| of its sum, u |z| each of sm_scale * log2(e) (two
roundings), of the product with it and of the difference to the reference: 8 u |z| are allowed.  A weight is off by that, by 2 u
of the hardware's power of two, and by u and less as three numbers: 4 u more.  Sums over n keys go through 3 n products and the joins
of four waves and of the two halves of the columns: 3 n + 10 roundings of sums that are no larger than the whole.
As two numbers a query or a weight would be off by up to 2^-17, 128 u.
"""
import numpy as np
import pytest
import torch

from test_gpu_kv4 import Problem, host, kv4  # noqa: F401  (kv4 is the fixture)

U = 2.0 ** -24


def two_numbers(x):
    """x as the sum of two bf16 numbers, each to nearest."""
    def bf16(a):
        return torch.from_numpy(np.ascontiguousarray(a)).to(torch.bfloat16).double().numpy()
    first = bf16(x)
    return first + bf16(x - first)


def attention(q, k, v, scale, short_queries=False, short_weights=False):
    """(out, lse, tolerance of out, tolerance of lse) of rows q [m, D] over the same keys and values [n, D], in 64 bits."""
    n = len(k)
    z = (two_numbers(q) if short_queries else q) @ k.T * scale
    top = z.max(axis=1, keepdims=True)
    w = np.exp(z - top)
    lse = (top + np.log(w.sum(axis=1, keepdims=True)))[:, 0]
    if short_weights:
        w = two_numbers(w)
    w = w / np.exp(z - top).sum(axis=1, keepdims=True)
    out = w @ v
    off = w * (8 * U * np.abs(z) + 4 * U)
    sums = (3 * n + 10) * U
    tol = off @ np.abs(v) + off.sum(axis=1, keepdims=True) * np.abs(out) + sums * (w @ np.abs(v) + np.abs(out)) + 2 * U * np.abs(out)
    return out, lse, tol, off.sum(axis=1) + sums + 4 * U * (1 + np.abs(lse))


def queries(rng, tokens, heads, D, size):
    q = np.zeros((tokens, heads, D), dtype=np.float32)
    at = rng.integers(0, D, (tokens, heads))
    np.put_along_axis(q, at[:, :, None], (size * rng.standard_normal((tokens, heads, 1))).astype(np.float32), axis=2)
    return q


@pytest.mark.parametrize("D", [64, 128])
def test_the_bounds_tell_two_numbers_from_three(D):
    """The mistakes that the bounds are there for, made in the definition (no GPU)."""
    rng = np.random.default_rng(D)
    missed = {"short_queries": 0, "short_weights": 0}
    for n in (2, 3, 5):
        k = rng.integers(-6, 7, (n, D)) / 2.0
        v = rng.standard_normal((n, D))
        q = queries(rng, 200, 1, D, 10.0)[:, 0].astype(np.float64)
        ref, ref_lse, tol, tol_lse = attention(q, k, v, D ** -0.5)
        for mistake in missed:
            out, lse, _, _ = attention(q, k, v, D ** -0.5, **{mistake: True})
            missed[mistake] += int((np.abs(out - ref) > tol).any(axis=1).sum())
            if mistake == "short_queries":
                assert (np.abs(lse - ref_lse) > tol_lse).sum() > 20, n
    assert missed["short_queries"] > 100 and missed["short_weights"] > 30, missed


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hkv,news", [(8, 1, 1), (7, 1, 1), (4, 2, 4), (4, 1, 4), (8, 1, 4), (8, 1, 8), (8, 1, 17), (1, 1, 40), (2, 2, 70)])
def test_few_keys_in_single_precision(kv4, H, Hkv, news, D):  # noqa: F811
    """Single tokens, drafts of up to 8, 16 and 32 rows, and chunks whose tiles have up to 64 rows and more: rows that see up to five
    keys of many requests."""
    requests = 60 if news < 10 else 12
    lens = [news + r % 5 for r in range(requests)]
    p = Problem(kv4, lens, [news] * requests, H, Hkv, D, 32, torch.float32, seed=D + news)
    p.q = torch.from_numpy(queries(np.random.default_rng(news), requests * news, H, D, 10.0)).cuda()
    out, lse, q = host(p.run()).astype(np.float64), host(p.lse).astype(np.float64), host(p.q).astype(np.float64)
    first, checked = np.concatenate([[0], np.cumsum(lens)]), 0
    for r in range(requests):
        for t in range(news):
            n = lens[r] - news + t + 1
            if n > 5:
                break
            for g in range(Hkv):
                at = int(p.start[r]) + t, slice(g * p.G, (g + 1) * p.G)
                ref, ref_lse, tol, tol_lse = attention(q[at], p.k[first[r]:first[r] + n, g], p.v[first[r]:first[r] + n, g], p.scale)
                assert np.all(np.abs(out[at] - ref) <= tol), (r, t, g, (np.abs(out[at] - ref) / tol).max())
                assert np.all(np.abs(lse[at] - ref_lse) <= tol_lse), (r, t, g)
                checked += 1
    assert checked >= 30
