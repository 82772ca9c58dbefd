"""The paged generation example end to end: its last step's attention against the same over the rows read back from the
cache, in 64 bits, and the pages that it gives back."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_paged_generation():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paged_generation as example
    last = example.generate(requests=3, steps=40, prompt=1500, shots=7, budget=500, q_heads=8, kv_heads=2, seed=3)
    cache, lens = last["cache"], last["lens"].tolist()
    assert lens == [n + 40 for n in last["in_cache"].tolist()] and not last["status"].any() and min(lens) > 40
    q, out, table = (last[x].float().cpu().numpy() for x in ("q", "out", "table"))
    for r, n in enumerate(lens):
        slots = table[r].astype(np.int64)[np.arange(n) // example.PAGE] * example.PAGE + np.arange(n) % example.PAGE
        k, v = (t.cpu().numpy().astype(np.float64) for t in
                example.kv4.load(cache, torch.from_numpy(slots.astype(np.int32)).cuda(), dtype=torch.float32))
        for g in range(2):
            ref, _, spread = orc.attention(q[r:r + 1, 4 * g:4 * g + 4], k[:, g], v[:, g], 1, last["scale"])
            # weights off by 2^-16, logits by 32-bit roundings, the output by one rounding to bf16
            assert np.all(np.abs(out[r:r + 1, 4 * g:4 * g + 4] - ref) <= 5e-5 * spread + 2.0 ** -8 * np.abs(ref))
    assert int(last["left"]) == cache.n_pages
    assert sorted(last["free"].tolist()) == list(range(cache.n_pages))
