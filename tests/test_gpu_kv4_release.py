"""Pages that are given back by requests whose rows are not all pages of their own."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from test_gpu_kv4 import check_plan, i32, kv4, run_plan  # noqa: F401  (kv4 is the fixture)

pytestmark = pytest.mark.gpu


def release(kv4, page, finished, lens, table, stack, count):  # noqa: F811
    """Results of a release on the GPU, checked against the definition."""
    got = [i32(lens), i32(table), i32(stack), i32([count])]
    kv4.pages_release(page, torch.from_numpy(np.asarray(finished, dtype=np.uint8)).cuda(), *got)
    want = orc.pages_release(page, np.asarray(finished), np.asarray(lens), np.asarray(table), np.asarray(stack), count)
    for g, w in zip(got, want):
        np.testing.assert_array_equal(g.cpu().numpy().reshape(np.shape(w)), w)
    return [np.asarray(w) for w in want]


@pytest.mark.parametrize("R,max_pages,missing", [(1, 1, 1.0), (3, 5, 0.5), (40, 70, 0.1), (70, 700, 0.02), (5, 1300, 0.5), (300, 9, 0.0)])
def test_entries_that_are_no_pages_do_not_reach_the_stack(kv4, R, max_pages, missing):  # noqa: F811
    rng = np.random.default_rng(R)
    lens = rng.integers(0, max_pages * 32 + 1, R)
    lens[0] = max_pages * 32
    total = int((-(-lens // 32)).sum())
    table, pool = np.full((R, max_pages), -1), rng.permutation(total + 10)
    for r in range(R):
        n = -(-lens[r] // 32)
        table[r, :n], pool = np.where(rng.random(n) < missing, -1 - rng.integers(0, 5, n), pool[:n]), pool[n:]
    stack = np.concatenate([rng.permutation(10) + 10**6, np.full(total, -77)])
    for finished in (np.ones(R, bool), rng.random(R) < 0.5):
        _, _, free, count = release(kv4, 32, finished, lens, table, stack, 10)
        assert (free[:int(count)] >= 0).all()


def test_requests_that_share_pages(kv4):  # noqa: F811
    """Two requests over a common prefix: the one that ends first leaves the prefix out, the other gives it back, and a plan after
    each hands every page to one owner."""
    page = 32
    table = np.array([[6, 7, 0, -1], [6, 7, 1, 2], [-1, -1, -1, -1]])
    lens, stack, count = np.array([90, 128, 0]), np.array([3, 4, 5, -77, -77, -77, -77, -77]), 3
    table[0, :2] = -1                   # still in use by the second request
    lens, table, stack, count = release(kv4, page, [1, 0, 0], lens, table, stack, count)
    assert sorted(stack[:int(count)]) == [0, 3, 4, 5] and table[1].tolist() == [6, 7, 1, 2]
    plan = run_plan(kv4, page, lens, [0, 0, 128], stack, int(count), table, 128)
    check_plan(plan, orc.pages_plan(page, lens, [0, 0, 128], stack, int(count), table, 128))
    table, lens, count = plan.block_table.cpu().numpy(), plan.seq_lens.cpu().numpy(), int(plan.free_left)
    assert sorted(table[1].tolist() + table[2].tolist()) == list(range(8)) and count == 0 and plan.status.tolist() == [0, 0, 0]
    lens, table, stack, count = release(kv4, page, [1, 1, 1], lens, table, stack, count)
    assert sorted(stack[:int(count)]) == list(range(8)) and not lens.any() and (table == -1).all()
