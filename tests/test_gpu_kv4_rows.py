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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H,Hkv,D,rot,interleaved", [
    (4096, 32, 8, 128, 128, False), (3001, 35, 7, 64, 64, False), (5000, 20, 5, 64, 32, True), (1537, 64, 8, 128, 128, True),
    (2111, 13, 13, 128, 64, False),                                         # in a group the last queries and the first keys
    (8200, 30, 6, 128, 128, False), (40001, 12, 4, 64, 64, False)])         # eight heads to a wave: fetched twice, of two kinds
def test_chunks_of_prompts_with_and_without_the_cache(kv4, T, H, Hkv, D, rot, interleaved, dtype):  # noqa: F811
    """Lengths at which a wave goes through several heads, of more than one kind: rows against the definition, and what the same
    pass stores against a store of its rows."""
    dt, page = TYPES[dtype], 64
    g = torch.Generator(device="cuda").manual_seed(T)
    qkv = (torch.randn((T, H + 2 * Hkv, D), generator=g, device="cuda") * torch.logspace(-3, 3, T, device="cuda")[:, None, None]).to(dt)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    rope = make_rope(kv4, D, rot, dt, interleaved, True, H)
    rng = np.random.default_rng(T)
    pos = rng.integers(0, 700, T)
    pos[[1, T // 2, T - 2]] = -1, 700, 2**31 - 1        # padding
    q_out, k_out = kv4.qk_norm_rope(rope, q, k, i32(pos))
    at = np.unique(np.r_[0:3, rng.integers(0, T, 12), T // 2, T - 3:T])
    here = torch.from_numpy(at).cuda()
    check_rotated(q_out[here], q[here], rope.q_weight, rope, pos[at], dt)
    check_rotated(k_out[here], k[here], rope.k_weight, rope, pos[at], dt)
    # a prompt by head
    by_head = [torch.full((n, T, D), 9.0, dtype=dt, device="cuda") for n in (H, Hkv)]
    kv4.qk_norm_rope(rope, q, k, i32(pos), by_head[0].transpose(0, 1), by_head[1].transpose(0, 1))
    assert torch.equal(by_head[0].transpose(0, 1), q_out) and torch.equal(by_head[1].transpose(0, 1), k_out)
    # and into the cache, with the keys as well and without
    n_pages = -(-T // page) + 3
    slots = rng.permutation(n_pages * page)[:T]
    slots[[0, T - 1]] = -1, n_pages * page
    kept = np.where((pos >= 0) & (pos < 700), slots, -1)
    pools = [torch.full((n_pages, kv4.page_bytes(page, Hkv, D)), 7, dtype=torch.uint8, device="cuda") for _ in range(3)]
    q2, k2 = kv4.qk_norm_rope(rope, q, k, i32(pos), None, None, v, kv4.Cache(pools[0], page, Hkv, D), i32(slots))
    q3, k3 = kv4.qk_norm_rope(rope, q, k, i32(pos), None, torch.empty_like(k_out), v, kv4.Cache(pools[1], page, Hkv, D), i32(slots))
    kv4.store(kv4.Cache(pools[2], page, Hkv, D), k_out, v, i32(kept))
    assert k2 is None and torch.equal(q2, q_out) and torch.equal(q3, q_out) and torch.equal(k3, k_out)
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[2])
