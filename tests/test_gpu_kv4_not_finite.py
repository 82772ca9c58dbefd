"""Values that are not finite in the paged 4-bit cache: every row that sees one is NaN in its group of 32 channels, however little
weight its key has, wherever it stands and whichever kernel takes the request; no other row and no other channel is."""
import numpy as np
import pytest
import torch

from test_gpu_kv4 import TYPES, Problem, host, kv4  # noqa: F401  (kv4 is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("news", [1, 3, 8, 12, 40, 100])
@pytest.mark.parametrize("length", [150, 3000])
def test_values_without_weight(kv4, length, news, D, dtype):  # noqa: F811
    """All weight is on one key (logits apart by more than 150): weights of the others are zero in 32 bits."""
    ends = length - news        # rows see keys up to ends + i
    for ahead, bad in ((5, 40), (40, 5), (8, 9), (9, 8), (ends // 2, ends // 2 - 33), (ends // 2 - 33, ends // 2), (5, ends - 1), (5, ends),
                       (ends, 5), (5, ends + news // 2), (ends - 1, ends + (news - 1) // 2), (33, length - 1)):
        if ahead == bad or ahead > ends or min(ahead, bad) < 0:
            continue

        def values(k, v):
            k[ahead], v[bad, :, 40:] = 6.0, np.inf
        p = Problem(kv4, [length], [news], 4, 1, D, 32, TYPES[dtype], values=values, seed=news)
        p.q.fill_(4.0)
        out, lse = host(p.run()), host(p.lse)
        sees = ends + np.arange(news) >= bad
        assert np.isfinite(lse).all(), (ahead, bad)
        assert np.isfinite(out[:, :, :32]).all() and np.isfinite(out[~sees]).all(), (ahead, bad)
        assert np.isnan(out[sees][:, :, 32:]).all(), (ahead, bad)
        np.testing.assert_array_equal(out[:, :, :32], np.broadcast_to(p.v[ahead, 0, :32].astype(np.float32), out[:, :, :32].shape))
