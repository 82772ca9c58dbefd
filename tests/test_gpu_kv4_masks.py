"""Which keys the queries of the paged 4-bit cache's attention see where a call's limits cut its requests."""
import numpy as np
import pytest
import torch

from test_gpu_kv4 import Problem, i32, kv4  # noqa: F401  (kv4 is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.float32)])
@pytest.mark.parametrize("lens,news,most", [
    ([70, 300, 40], [2, 3, 1], 2), ([70, 300, 40], [2, 3, 1], 1), ([500, 33, 64], [9, 33, 5], 4), ([5, 400, 2], [7, 200, 1], 3),
    ([400, 90, 700], [150, 90, 300], 70), ([3000, 31], [130, 40], 100)])
def test_a_request_cut_to_max_q_len_keeps_its_mask(kv4, lens, news, most, D, dtype):  # noqa: F811
    """The first max_q_len tokens of a longer request see what they see in a call that takes all of it; those after them are left
    as they were."""
    p = Problem(kv4, lens, news, 8, 2, D, 32, dtype, seed=most)
    p.check(p.run())
    out, lse = torch.full_like(p.q, 5.0), torch.full((len(p.q), 8), 5.0, device="cuda")
    kv4.attention(p.cache, p.q, p.table, i32(p.lens), p.scale, i32(p.start), most, out, lse)
    for r, n in enumerate(news):
        first, cut = int(p.start[r]), min(n, most)
        assert torch.all(out[first + cut:first + n] == 5) and torch.all(lse[first + cut:first + n] == 5), r
        # the taken tokens are those of a request that ends with them
        q = Problem.__new__(Problem)
        q.__dict__.update(p.__dict__)
        end = lens[r] - (n - cut)
        q.lens, q.news, q.start = [max(end, 0)], [cut], [0, cut]
        at = sum(lens[:r])
        q.k, q.v, q.q = p.k[at:at + max(end, 0)], p.v[at:at + max(end, 0)], p.q[first:first + cut]
        if end >= 0:
            q.check(out[first:first + cut], lse[first:first + cut])
        else:
            assert not out[first:first + cut].any() and torch.all(torch.isneginf(lse[first:first + cut]))


@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.float32)])
@pytest.mark.parametrize("requests", [70, 300])
def test_chunks_of_many_requests(kv4, requests, D, dtype):  # noqa: F811
    """More requests than a wave has lanes, and than a workgroup has threads: chunks of some, single tokens of others, none of a few."""
    rng = np.random.default_rng(requests)
    news = rng.integers(0, 40, requests)
    news[::3] = 1
    lens = news + rng.integers(0, 60, requests)
    p = Problem(kv4, lens, news, 8, 2, D, 32, dtype, seed=requests)
    p.check(p.run())
