"""Drafts of requests that a tree plan refuses: their rows were not stored and nobody's bits name them, so none of them is kept, their
requests stay as long as they were and their pages go back.  Whole numbers and bytes: equal."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from test_gpu_kv4 import i32, kv4  # noqa: F401  (kv4 is the fixture)
from test_gpu_kv4_tree import Drafted, Generation, make_trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_cache", [True, False])
@pytest.mark.parametrize("D,layers", [(128, 1), (64, 3)])
@pytest.mark.parametrize("news", [[5], [5, 7, 1, 0, 40], [70, 3, 66, 2], [1030, 4, 1025], [3] * 70])
def test_refused_requests_keep_nothing(kv4, news, D, layers, with_cache):  # noqa: F811
    """Any status but 0 refuses, of every request and of some; the others are kept as without one."""
    for refused in ([0], range(0, len(news), 2), range(len(news)), []):
        d = Drafted(kv4, news, 2, D, layers=layers, luck=0.9, seed=len(news))
        status = np.zeros(len(news), dtype=np.int64)
        for i, r in enumerate(refused):
            status[r] = (-6, -5, 1, 2**31 - 1, -2**31, 256)[i % 6]
        kept = kv4.TreeKept.empty(d.R, max(news))
        for t in (kept.path, kept.accepted, kept.next_token):
            t.fill_(-77)
        before = d.cache.pages.cpu().numpy().reshape(-1).copy()
        lens = kept.kept_lens = i32(d.lens)     # in place
        n_slots = d.per_layer * d.page
        args = (d.cache, i32(d.slots), layers) if with_cache else ()
        kv4.tree_keep(i32(d.start), i32(d.parents), i32(d.tokens), i32(d.chosen), lens, kept, *args, status=i32(status))
        path, accepted, following, kept_lens, moves = orc.tree_keep(d.start, d.parents, d.tokens, d.chosen, d.lens, max(news),
                                                                    d.slots if with_cache else None, n_slots, status)
        for name, want in (("path", path), ("accepted", accepted), ("next_token", following), ("kept_lens", kept_lens)):
            np.testing.assert_array_equal(getattr(kept, name).cpu().numpy(), want, err_msg=name)
        for r in refused:
            assert not accepted[r] and following[r] == -1 and (path[r] == -1).all() and kept_lens[r] == d.lens[r]
        for layer in range(layers):
            for source, target in moves:
                orc.move(before, d.page, d.Hkv, D, source + layer * n_slots, target + layer * n_slots)
        np.testing.assert_array_equal(d.cache.pages.cpu().numpy().reshape(-1), before)


@pytest.mark.parametrize("with_cache", [True, False])
def test_a_step_with_trees_that_are_refused(kv4, with_cache):  # noqa: F811
    """Plan, tree plan, rotation and store, keep, trim: a tree with a parent that is not before its token, one of more drafts than the
    plan has bits for, and a sound one."""
    rng = np.random.default_rng(0)
    page, Hkv, D, news, cached = 32, 2, 128, [9, 40, 12], [50, 64, 31]
    T, start = sum(news), [0, 9, 49, 61]
    parents = make_trees(rng, news)
    parents[[0, 9, 49]] = -1
    parents[4] = 4
    tokens = np.arange(T)
    chosen = np.full(T, -1)
    for first, n in zip(start, news):       # every first child is chosen
        for i in range(n - 1, 0, -1):
            if 0 <= parents[first + i] < i:
                chosen[first + parents[first + i]] = tokens[first + i]
    table = np.full((3, 6), -1)
    table[0, :2], table[1, :2], table[2, :1] = [0, 1], [2, 3], [4]
    pages = torch.from_numpy(rng.integers(0, 256, (20, kv4.page_bytes(page, Hkv, D)), dtype=np.uint8)).cuda()
    cache, free, count = kv4.Cache(pages, page, Hkv, D), i32(np.arange(5, 20)), i32([15])
    plan, tree, kept = kv4.PagePlan.empty(i32(table), T), kv4.TreePlan.empty(3, T, 32), kv4.TreeKept.empty(3, 12)
    lens = i32(cached)
    kept.kept_lens = lens
    before, stack = pages.clone(), free.clone()
    kv4.pages_plan(page, lens, i32(news), free, count, plan)
    assert plan.status.tolist() == [0, 0, 0] and (plan.slot_map >= 0).all()     # all have their pages
    kv4.tree_plan(plan.query_start, i32(parents), lens, tree)
    assert tree.status.tolist() == [-6, -5, 0] and (tree.token_pos[:49] == -1).all() and not tree.tree_mask[:49].any()
    rope = kv4.Rope(torch.ones((200, D), device="cuda"))
    q, k, v = (torch.from_numpy(rng.standard_normal((T, h, D))).bfloat16().cuda() for h in (4, Hkv, Hkv))
    kv4.qk_norm_rope(rope, q, k, tree.token_pos, v=v, cache=cache, slot_map=plan.slot_map)
    stored = pages.clone()
    args = (cache, plan.slot_map) if with_cache else ()
    kv4.tree_keep(plan.query_start, i32(parents), i32(tokens), i32(chosen), lens, kept, *args, status=tree.status)
    accepted = kept.accepted.tolist()
    assert accepted[:2] == [0, 0] and accepted[2] >= 2
    assert lens.tolist() == [50, 64, 31 + accepted[2]] and kept.next_token.tolist()[:2] == [-1, -1] and (kept.path[:2] == -1).all()
    theirs = [p for p in range(20) if p not in plan.block_table[2].tolist()]
    assert torch.equal(pages[theirs], before[theirs]) and not torch.equal(stored, before)       # nothing of theirs was written
    left, given = i32([0]), i32(np.zeros(3))
    kv4.pages_trim(page, plan.seq_lens, lens, plan.block_table, free, plan.free_left, left, given)
    assert plan.block_table[0].tolist() == [0, 1, -1, -1, -1, -1] and plan.block_table[1].tolist() == [2, 3, -1, -1, -1, -1]
    used = plan.block_table[plan.block_table >= 0].tolist()
    assert sorted(used + free[:int(left)].tolist()) == list(range(20)) and len(stack) == 15


def test_refused_trees_in_a_graph(kv4):  # noqa: F811
    """A captured step whose trees are refused in some replays: those requests stay as they were and go on with the next."""
    g = Generation(kv4, seed=9)
    g.take(g.inputs(0))
    keep = g.kv4.tree_keep

    class Planned:      # the step's own calls, with the plan's status at the one
        def __getattr__(self, name):
            return getattr(kv4, name)

        def tree_keep(self, *args):
            return keep(*args, status=g.tree.status)
    g.kv4 = Planned()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g.step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.step()
    for i in range(1, 12):
        drafts = g.inputs(i)
        bad = [r for r in range(g.R) if (r + i) % 3 == 0]
        for r in bad:
            drafts[0][r * g.nodes + 5] = 7 + i
        g.take(drafts)
        before = g.lens.tolist()
        graph.replay()
        assert [r for r, s in enumerate(g.tree.status.tolist()) if s] == bad
        for r, n in enumerate(g.lens.tolist()):
            assert (n == before[r]) if r in bad else (n > before[r]), (i, r)
        held = g.table[g.table >= 0].tolist()
        assert sorted(held + g.free[:int(g.count)].tolist()) == list(range(g.per_layer))


def test_refusals(kv4):  # noqa: F811
    start, ints, lens, kept = i32([0, 3]), i32([0, 0, 0]), i32([5]), kv4.TreeKept.empty(1, 3)
    for bad, why in ((i32([0, 0]), "shape"), (torch.zeros(1, device="cuda"), "int32"), (torch.zeros(1, dtype=torch.int32), "GPU")):
        with pytest.raises(kv4.ShotKVError, match=why):
            kv4.tree_keep(start, ints, ints, ints, lens, kept, status=bad)
