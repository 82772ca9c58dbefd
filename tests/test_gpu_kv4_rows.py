"""Norms and rotation of the paged 4-bit cache at sizes and lengths that a prompt has.  Tolerances as in test_gpu_kv4."""
import numpy as np
import pytest
import torch

from test_gpu_kv4 import TYPES, check_rotated, i32, kv4, make_rope  # noqa: F401  (kv4 is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,interleaved", [(64, False), (128, False), (128, True)])
def test_norms_of_rows_of_any_size(kv4, D, interleaved, dtype):  # noqa: F811
    """Rows whose squares overflow or vanish in 32 bits, next to ordinary ones, with and without an epsilon."""
    sizes = np.concatenate([10.0 ** np.arange(-37, 38), [3e37, 2e-38, 1.0, 0.0]])
    g = torch.Generator().manual_seed(D)
    x = torch.randn((len(sizes), 3, D), generator=g, dtype=torch.float64) * torch.from_numpy(sizes)[:, None, None]
    x = x.to(TYPES[dtype]).cuda()
    both = make_rope(kv4, D, D, TYPES[dtype], interleaved, True, D)
    pos = np.arange(len(sizes))
    for eps in (1e-5, 1e-25, 0.0):
        rope = kv4.Rope(both.table, both.q_weight, both.k_weight, eps, interleaved)
        keep = len(sizes) - (eps == 0)          # (a row of zeros without an epsilon is 0 / 0)
        q, k = kv4.qk_norm_rope(rope, x[:keep, :2], x[:keep, 2:], i32(pos[:keep]))
        check_rotated(q, x[:keep, :2], rope.q_weight, rope, pos, TYPES[dtype])
        check_rotated(k, x[:keep, 2:], rope.k_weight, rope, pos, TYPES[dtype])
