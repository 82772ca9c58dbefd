"""Bytes that nobody stored where a row does not look: behind a window, between sinks and window, and in drafts of other branches.  A row's
result goes by the tokens that it sees, whatever the bytes of the others are.

A store writes scale bytes up to 252, and 255.  253 and 254 stand for 2^126 and 2^127: with codes of 4 and more (2 and more) numbers past the
largest one that bf16 holds, 2^128 - 2^120.  Such a number is infinite as a factor, and an infinity times a weight of zero is NaN.

Tolerances are those of test_gpu_kv4_seen: the rows that are compared see nothing that is out of the ordinary.
"""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from test_gpu_kv4 import TYPES, host, kv4  # noqa: F401  (kv4 is the fixture)
from test_gpu_kv4_seen import Seen

pytestmark = pytest.mark.gpu

# (scale byte, byte of two codes): 6 and -6, 4, 2, 3 (a number that bf16 holds, next to the largest), the largest that is stored, NaN
BYTES = [(254, 0x77), (254, 0xff), (253, 0x66), (253, 0xef), (254, 0x44), (253, 0x55), (252, 0x77), (255, 0x77)]
PAST = BYTES[:5]        # past the largest number of bf16
SHAPES = [(8, 2, [700, 33, 400], [1, 1, 1]), (8, 2, [700, 33, 400], [2, 2, 3]), (8, 2, [700, 33, 200], [8, 2, 3]), (4, 1, [300, 90, 700], [16, 12, 9]),
          (8, 2, [700, 64, 130], [100, 12, 20])]


def fill(p, at, scale, codes, keys=True, groups=None):
    """The bytes of tokens `at` of the problem (numbers in its list of slots), of all groups of 32 channels or of some."""
    page, D = p.cache.page_size, p.D
    pool = p.cache.pages.cpu().numpy().reshape(-1)
    for slot in p.slots[at]:
        for head in range(p.Hkv):
            key, values, key_scales, value_scales = orc._places(page, p.Hkv, D, int(slot), head)
            if keys:
                pool[key:key + D // 2] = codes
                pool[key_scales:key_scales + D // 32] = scale
            for g in range(D // 32) if groups is None else groups:
                for c in range(4 * g, 4 * g + 4):
                    pool[values[c]:values[c] + 4] = codes
                pool[value_scales[g]] = scale
    p.cache.pages.copy_(torch.from_numpy(pool.reshape(p.cache.pages.shape)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,window,sinks", [(None, 50, 3), (None, 1, 0), (None, 130, 40), ("tree", 50, 3), ("any", 90, 0), ("tree", 0, 0)])
@pytest.mark.parametrize("shape", SHAPES)
def test_tokens_that_nobody_sees_may_be_any_bytes(kv4, shape, kind, window, sinks, D, dtype):  # noqa: F811
    H, Hkv, lens, news = shape
    p = Seen(kv4, lens, news, H, Hkv, D, 64, TYPES[dtype], seed=D + news[0]).set(window, sinks, kind, seed=sum(news))
    unseen = np.concatenate([~p.seen(r).any(axis=0) for r in range(len(lens))])
    assert unseen.any() or (kind == "tree" and not window)
    for scale, codes in BYTES:
        fill(p, np.flatnonzero(unseen), scale, codes)
        p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", [None, "tree", "any"])
@pytest.mark.parametrize("news", [2, 3, 8, 14, 40, 100])
def test_tokens_that_some_rows_see(kv4, kind, news, D, dtype):  # noqa: F811
    """The second group of 32 channels of a token's values: the rows that do not see the token are right, the others in all other groups."""
    length, window = 300, 90
    for at in (length - news - window + 1, length - news - window + news // 2, length - news, length - news + news // 2):
        p = Seen(kv4, [length], [news], 4, 1, D, 32, TYPES[dtype], seed=news).set(window if kind != "tree" else 0, 0, kind, seed=news)
        q = host(p.q).astype(np.float64)
        seen = p.seen(0)
        sees = seen[:, at]
        ref, _, spread = orc.seen_attention(q, p.k[:, 0], p.v[:, 0], seen, p.scale)
        tol = 5e-5 * spread + (np.abs(ref) * 2.0 ** -8 if p.dtype == torch.bfloat16 else 0)
        for scale, codes in BYTES:
            fill(p, [at], scale, codes, keys=False, groups=[1])
            out, lse = host(p.run()), host(p.lse)
            assert np.isfinite(lse[seen.any(axis=1)]).all(), (at, scale, codes)
            right = np.abs(out - ref) <= tol
            assert right[~sees].all(), (at, scale, codes)
            assert right[sees][:, :, :32].all() and right[sees][:, :, 64:].all(), (at, scale, codes)
            if (scale, codes) in PAST:
                assert not np.isfinite(out[sees][:, :, 32:64]).any(), (at, scale, codes)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("news", [2, 14, 100])
def test_one_number_past_the_largest(kv4, news, dtype):  # noqa: F811
    """A group with one code that is too large for its scale, the others zero, beside tokens that all rows see."""
    length, window = 300, 90
    at = length - news - window + news // 2
    for D in (64, 128):
        p = Seen(kv4, [length], [news], 4, 1, D, 32, TYPES[dtype], seed=news).set(window)
        fill(p, [at], 254, 0, keys=False, groups=[1])
        p.v[at, 0, 32:64] = 0.0         # a scale by itself is no number
        p.check(p.run())
        pool = p.cache.pages.cpu().numpy().reshape(-1)
        pool[orc._places(32, 1, D, int(p.slots[at]), 0)[1][5]] = 0x40       # 2 in channel 41
        p.cache.pages.copy_(torch.from_numpy(pool.reshape(p.cache.pages.shape)))
        sees = p.seen(0)[:, at]
        assert sees.any() and not sees.all()
        out = host(p.run())
        assert not np.isfinite(out[sees][:, :, 41]).any() and np.isfinite(out[~sees]).all()
        ref, _, spread = orc.seen_attention(host(p.q).astype(np.float64), p.k[:, 0], p.v[:, 0], p.seen(0), p.scale)
        tol = 5e-5 * spread + (np.abs(ref) * 2.0 ** -8 if p.dtype == torch.bfloat16 else 0)
        right = np.abs(out - ref) <= tol
        assert right[~sees].all() and right[sees][:, :, :32].all() and right[sees][:, :, 64:].all()
