"""Trees of drafts around the paged 4-bit cache - what they see, which of them stay, pages that go back - against plain
definitions, through the public binding.  All results are whole numbers or bytes: equal."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from test_gpu_kv4 import i32, kv4  # noqa: F401

pytestmark = pytest.mark.gpu


def make_trees(rng, news, kind="tree"):
    parents = []
    for n in news:
        for i in range(n):
            parents.append(-int(rng.integers(1, 9)) if i == 0 or rng.random() < 0.05 else i - 1 if kind == "chain" else int(rng.integers(0, i)))
    return np.array(parents, dtype=np.int64).reshape(-1)


# ---- plans -----------------------------------------------------------------------------------------------

def run_plan(kv4, start, parents, pos, words):  # noqa: F811
    T, R = len(parents), len(start) - 1
    plan = kv4.TreePlan.empty(R, T, 32 * words)
    assert plan.tree_mask.shape == (T, words)
    for t in (plan.tree_mask, plan.token_pos, plan.status):
        t.fill_(-77)
    kv4.tree_plan(i32(start), i32(parents), i32(pos), plan)
    return plan


def check_plan(plan, ref):
    mask, pos, status = ref
    np.testing.assert_array_equal(plan.tree_mask.cpu().numpy().view(np.uint32), mask.astype(np.uint32))
    np.testing.assert_array_equal(plan.token_pos.cpu().numpy(), pos)
    np.testing.assert_array_equal(plan.status.cpu().numpy(), status)


@pytest.mark.parametrize("kind", ["tree", "chain"])
@pytest.mark.parametrize("R,most,words", [(1, 1, 1), (16, 5, 1), (7, 32, 1), (5, 33, 2), (300, 64, 2), (3, 256, 8), (4, 300, 10), (2, 1024, 32),
                                          (9, 20, 32), (40, 130, 5), (6, 1024, 32)])
def test_tree_plan(kv4, R, most, words, kind):  # noqa: F811
    rng = np.random.default_rng(R + most)
    news = rng.integers(0, most + 1, R)
    news[0] = most
    parents, start = make_trees(rng, news, kind), np.concatenate([[0], np.cumsum(news)])
    pos = rng.integers(0, 100000, R)
    check_plan(run_plan(kv4, start, parents, pos, words), orc.tree_plan(start, parents, pos, words))


def test_tree_plan_says_what_is_wrong(kv4):  # noqa: F811
    """Parents that are not before their tokens, too many drafts, starts outside the batch, positions past 31 bits, rows of nobody."""
    rng = np.random.default_rng(1)
    news = [5, 40, 3, 33, 0, 6]
    parents = make_trees(rng, news)
    parents[2], parents[45 + 2], parents[81 + 5] = 2, 2**31 - 1, 4
    start = np.concatenate([[0], np.cumsum(news)])
    pos = [7, 8, 9, 10, 11, 2**31 - 2]
    ref = orc.tree_plan(start, parents, pos, 1)
    assert ref[2].tolist() == [-6, -5, -6, -5, 0, 0]
    check_plan(run_plan(kv4, start, parents, pos, 1), ref)
    check_plan(run_plan(kv4, start, parents, pos, 2), orc.tree_plan(start, parents, pos, 2))
    for odd in ([2, 5, 45, 40, 81, 85, 10**6], [-5, 5, 45, 48, 81, 81, 86], [90, 90, 90, 90, 90, 90, 90], [87, 60, 50, 40, 30, 20, 10]):
        mask, at, status = orc.tree_plan(odd, parents, pos, 2)
        got = run_plan(kv4, odd, parents, pos, 2)
        np.testing.assert_array_equal(got.status.cpu().numpy(), status)
        if all(a <= b for a, b in zip(odd, odd[1:])):       # (of starts that fall, requests share rows)
            check_plan(got, (mask, at, status))


# ---- keeping ---------------------------------------------------------------------------------------------

class Drafted:
    """Requests with drafts in pages of `layers` layers of a pool, all bytes random."""

    def __init__(self, kv4, news, Hkv=2, D=128, page=32, layers=1, seed=0, kind="tree", luck=0.8, ids=50):  # noqa: F811
        rng = np.random.default_rng(seed)
        self.R, self.T = len(news), int(np.sum(news))
        self.start = np.concatenate([[0], np.cumsum(news)])
        self.parents = make_trees(rng, news, kind)
        self.tokens, self.chosen = rng.integers(0, ids, self.T), rng.integers(0, ids, self.T)
        index = np.concatenate([np.arange(n) for n in news]) if self.T else np.zeros(0, int)
        for t in np.nonzero(rng.random(self.T) < luck)[0]:
            if 0 <= self.parents[t] < index[t]:
                self.chosen[t - index[t] + self.parents[t]] = self.tokens[t]
        self.lens = rng.integers(0, 100, self.R)
        self.per_layer = self.T // page + self.R + 3
        self.slots = rng.permutation(self.per_layer * page)[:self.T]
        self.layers, self.page, self.Hkv, self.D = layers, page, Hkv, D
        pool = rng.integers(0, 256, (layers * self.per_layer, orc.page_bytes(page, Hkv, D)), dtype=np.uint8)
        self.cache = kv4.Cache(torch.from_numpy(pool).cuda(), page, Hkv, D)
        self.kv4 = kv4

    def check(self, max_path, with_cache=True, in_place=False):
        kept = self.kv4.TreeKept.empty(self.R, max_path)
        for t in (kept.path, kept.accepted, kept.next_token, kept.kept_lens):
            t.fill_(-77)
        before, lens = self.cache.pages.cpu().numpy().copy(), i32(self.lens)
        if in_place:
            kept.kept_lens = lens
        args = (i32(self.start), i32(self.parents), i32(self.tokens), i32(self.chosen), lens, kept)
        n_slots = self.per_layer * self.page
        slots = self.slots if with_cache else None
        if with_cache:
            self.kv4.tree_keep(*args, self.cache, i32(self.slots), self.layers)
        else:
            self.kv4.tree_keep(*args)
        path, accepted, following, kept_lens, moves = orc.tree_keep(self.start, self.parents, self.tokens, self.chosen, self.lens, max_path,
                                                                    slots, n_slots)
        for name, want in (("path", path), ("accepted", accepted), ("next_token", following), ("kept_lens", kept_lens)):
            np.testing.assert_array_equal(getattr(kept, name).cpu().numpy(), want, err_msg=name)
        want = before.reshape(-1).copy()
        for layer in range(self.layers):
            for source, target in moves:
                orc.move(want, self.page, self.Hkv, self.D, source + layer * n_slots, target + layer * n_slots)
        np.testing.assert_array_equal(self.cache.pages.cpu().numpy().reshape(-1), want)
        return accepted, moves


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("kind", ["tree", "chain"])
@pytest.mark.parametrize("news,Hkv,layers", [([1], 1, 1), ([5, 0, 1, 7], 2, 1), ([64, 33, 20, 16], 8, 1), ([65, 128, 3], 3, 2), ([300, 257, 40], 5, 3),
                                             ([16] * 40, 8, 4)])
def test_tree_keep(kv4, news, Hkv, layers, kind, D):  # noqa: F811
    for luck, ids in ((0.9, 50), (0.3, 3), (0.0, 1)):       # long paths, several children of one id, all of one id
        for max_path in (max(news), 3, 400):
            d = Drafted(kv4, news, Hkv, D, layers=layers, kind=kind, luck=luck, ids=ids, seed=sum(news))
            d.check(max_path, in_place=max_path == 3)
    assert d.check(max(news), with_cache=False)[0].max() >= 1


def test_long_paths_move_every_row(kv4):  # noqa: F811
    """Chains with a refused sibling at each step: every row of the path but the first moves, over more rows than a wave has lanes."""
    n = 401
    d = Drafted(kv4, [n, n], 2, 64, 64)
    i = np.arange(n)
    one = np.where(i % 2 == 0, i - 2, i - 1)        # 2, 4, 6, ... the chain; 1, 3, 5, ... children that nobody chose
    one[0] = -1
    d.parents, d.tokens, d.chosen = np.tile(one, 2), np.tile(i % 2, 2), np.zeros(2 * n, int)
    accepted, moves = d.check(300)
    assert accepted.tolist() == [201, 201] and len(moves) == 400


def test_more_drafts_than_a_mask_has_bits(kv4):  # noqa: F811
    """Requests of over 1024 drafts beside smaller ones: paths of any length, children far behind their parents."""
    for kind, luck, ids in (("tree", 0.9, 50), ("chain", 0.99, 5), ("tree", 0.0, 1)):
        for news in ([1024, 1025, 7], [3000, 1, 1030]):
            d = Drafted(kv4, news, 2, 64, 64, kind=kind, luck=luck, ids=ids, seed=len(kind))
            d.check(max(news))


def test_tree_keep_of_odd_calls(kv4):  # noqa: F811
    """Ids below 0 choose nothing, parents that are not before their tokens have no such children, slots outside of a layer stay."""
    d = Drafted(kv4, [6, 6, 6, 0, 6], 2, 128, layers=2, luck=1.0, seed=5)
    d.parents = np.tile([-1, 0, 1, 2, 3, 4], 4)
    d.tokens, d.chosen = np.tile([9, 1, 2, 3, 4, 5], 4), np.tile([1, 2, 3, 4, 5, 6], 4)
    d.chosen[2], d.tokens[3] = -1, -1
    d.parents[6 + 3] = 3
    d.parents[12:18] = [-1, 5, 0, 2, 2**31 - 1, -2**31]
    d.tokens[14] = 1
    d.chosen[14] = 3
    n_slots = d.per_layer * d.page
    d.slots[18], d.slots[19] = n_slots, -1          # the last request's first token has none
    accepted, _ = d.check(6)
    assert accepted.tolist() == [3, 3, 3, 0, 0]
    d.slots[18], d.slots[19], d.slots[15] = d.slots[20], n_slots + 5, -2**31     # a place in the path, and a row that would move
    d.check(6)
    d.start = np.array([3, 9, 9, 20, 24, 10**6])
    d.check(6)
    d.start = np.array([3, 9, -4, 20, 24, 10**6])       # (requests share drafts: nothing moves)
    d.check(6, with_cache=False)
    d = Drafted(kv4, [0, 0])
    d.check(4)


def test_tree_keep_in_a_pool_of_more_than_4_gib(kv4):  # noqa: F811
    """Two layers of a pool of 5 GiB: the second one's rows lie past 32 bits."""
    D, H, page = 128, 8, 128
    n_pages = 5 * 2**30 // kv4.page_bytes(page, H, D) // 2 * 2
    cache = kv4.Cache.empty(n_pages, page, H, D)
    half = n_pages // 2
    slots = (half - 1) * page + np.array([3, 50, 90, 127])
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = torch.randn((2, 8, H, D), generator=g, device="cuda")
    both = i32(np.concatenate([slots, slots + half * page]))
    kv4.store(cache, k, v, both)
    before = kv4.load(cache, both, dtype=torch.float32)
    kept = kv4.TreeKept.empty(1, 4)
    kv4.tree_keep(i32([0, 4]), i32([-1, 0, 0, 2]), i32([1, 2, 3, 4]), i32([3, 0, 4, 7]), i32([10]), kept, cache, i32(slots), 2)
    assert kept.path.tolist() == [[0, 2, 3, -1]] and kept.next_token.tolist() == [7] and kept.kept_lens.tolist() == [13]
    after = kv4.load(cache, both, dtype=torch.float32)
    for a, b in zip(before, after):
        assert torch.equal(b, a[[0, 2, 3, 3, 4, 6, 7, 7]])


# ---- pages that go back ----------------------------------------------------------------------------------

@pytest.mark.parametrize("R,page,most,window,sinks", [
    (1, 32, 500, None, 0), (16, 64, 700, None, 0), (16, 64, 700, 1, 0), (7, 32, 3000, 100, 4), (300, 32, 900, 64, 33), (300, 64, 2000, 333, 0),
    (5, 128, 90000, 1000, 200), (2, 32, 100000, 31, 32), (600, 32, 90, 32, 31), (64, 32, 900, 100, 4), (64, 32, 6000, 100, 4),
    (64, 32, 6000, None, 0), (65, 32, 900, None, 0), (1, 32, 200000, 3, 0), (3, 32, 900000, None, 0)])
def test_trim(kv4, R, page, most, window, sinks):  # noqa: F811
    rng = np.random.default_rng(R + page + most)
    held = rng.integers(0, most + 1, R)
    lens = np.maximum(held - rng.integers(0, 100, R), 0)
    lens[::5], held[::7] = held[::5], held[::7] // page * page
    columns = -(-max(int(held.max()), 1) // page) + 1
    table = rng.permutation(R * columns).reshape(R, columns)
    table[rng.random(table.shape) < 0.1] = -1       # gone before
    for size, count in ((R * columns + 10, 7), (R * columns, 0), (R * columns // 2, 5), (3, 3), (40, 1000), (40, -2)):
        free = np.arange(10**6, 10**6 + size)
        want = orc.pages_trim(page, held, lens, table, free, count, window or 0, sinks)
        got_table, got_free = i32(table), i32(free)
        left, given = i32([-77]), i32(np.full(R, -77))
        kv4.pages_trim(page, i32(held), i32(lens), got_table, got_free, i32([count]), left, given, window, sinks)
        np.testing.assert_array_equal(got_table.cpu().numpy(), want[0])
        np.testing.assert_array_equal(got_free.cpu().numpy(), want[1])
        assert int(left) == want[2]
        np.testing.assert_array_equal(given.cpu().numpy(), want[3])


def test_trim_of_lengths_that_make_no_sense(kv4):  # noqa: F811
    table = np.arange(48).reshape(8, 6)
    held, lens = [192, 192, -5, 10, 2**31 - 1, 2**31 - 1, 0, 100], [-3, 2**31 - 1, 4, 500, 0, 2**31 - 1, 0, -2**31]
    for window, sinks in ((None, 0), (40, 4), (2**30, 0), (1, 2**31 - 1)):
        want = orc.pages_trim(32, held, lens, table, np.zeros(60, int), 3, window or 0, sinks)
        got, free, left, given = i32(table), i32(np.zeros(60)), i32([0]), i32(np.zeros(8))
        kv4.pages_trim(32, i32(held), i32(lens), got, free, i32([3]), left, given, window, sinks)
        np.testing.assert_array_equal(got.cpu().numpy(), want[0])
        np.testing.assert_array_equal(free.cpu().numpy(), want[1])
        assert int(left) == want[2] and given.tolist() == want[3].tolist()


def test_a_trim_of_everything_undoes_a_plan(kv4):  # noqa: F811
    rng = np.random.default_rng(4)
    R, page = 90, 32
    new, stack = rng.integers(0, 200, R), rng.permutation(900)
    plan = kv4.PagePlan.empty(i32(np.full((R, 8), -1)), int(new.sum()))
    free, zeros = i32(stack), i32(np.zeros(R))
    kv4.pages_plan(page, zeros, i32(new), free, i32([900]), plan)
    left, given = i32([0]), i32(np.zeros(R))
    kv4.pages_trim(page, plan.seq_lens, zeros, plan.block_table, free, plan.free_left, left, given)
    np.testing.assert_array_equal(free.cpu().numpy(), stack)
    assert int(left) == 900 and torch.all(plan.block_table == -1) and given.tolist() == (-(-new // page)).tolist()


# ---- a run of them together ------------------------------------------------------------------------------

class Generation:
    """Steps of generation with drafted trees and a window, on static buffers, as a captured program would have them."""

    def __init__(self, kv4, R=5, nodes=13, window=70, sinks=4, dtype=torch.bfloat16, H=8, Hkv=2, D=128, page=32, layers=2, seed=0):  # noqa: F811
        rng = np.random.default_rng(seed)
        self.kv4, self.R, self.nodes, self.window, self.sinks, self.layers, self.H, self.Hkv, self.D, self.page = \
            kv4, R, nodes, window, sinks, layers, H, Hkv, D, page
        self.dtype, T, self.scale = dtype, R * nodes, 0.1
        self.per_layer, columns = R * 10, 40
        self.pages = torch.full((layers * self.per_layer, kv4.page_bytes(page, Hkv, D)), 255, dtype=torch.uint8, device="cuda")
        self.cache = kv4.Cache(self.pages, page, Hkv, D)
        self.layer_cache = [kv4.Cache(self.pages[i * self.per_layer:(i + 1) * self.per_layer], page, Hkv, D) for i in range(layers)]
        self.table = i32(np.full((R, columns), -1))
        self.plan = kv4.PagePlan.empty(self.table, T)
        self.tree = kv4.TreePlan.empty(R, T, nodes)
        self.kept = kv4.TreeKept.empty(R, nodes)
        self.free, self.count = i32(rng.permutation(self.per_layer)), i32([self.per_layer])
        self.left, self.given = i32([0]), i32(np.zeros(R))
        self.lens, self.new = i32(np.zeros(R)), i32(np.full(R, nodes))
        self.position = i32(np.arange(R) * 100)
        self.kept.kept_lens = self.lens
        angle = rng.uniform(0, 6.28, (4000, D // 2))
        self.rope = kv4.Rope(torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], axis=1)).float().cuda())
        self.parents, self.tokens, self.chosen = (i32(np.zeros(T)) for _ in range(3))
        self.qkv = torch.zeros((layers, T, H + 2 * Hkv, D), dtype=dtype, device="cuda")
        self.q = torch.zeros((layers, T, H, D), dtype=dtype, device="cuda")
        self.out = torch.zeros_like(self.q)
        self.ws = kv4.tree_attention_workspace(self.cache, self.q[0], self.table, nodes, window, sinks)

    def inputs(self, seed):
        """Drafts of a step: random trees, some of whose tokens the model chooses."""
        rng = np.random.default_rng(seed)
        T = self.R * self.nodes
        parents = np.concatenate([[-1] + [int(rng.integers(0, i)) for i in range(1, self.nodes)] for _ in range(self.R)])
        tokens, chosen = rng.integers(0, 1000, T), rng.integers(0, 1000, T)
        for t in np.nonzero((parents >= 0) & (rng.random(T) < 0.7))[0]:
            chosen[t - t % self.nodes + parents[t]] = tokens[t]
        qkv = torch.from_numpy(rng.standard_normal(tuple(self.qkv.shape))).to(self.dtype).cuda()
        return i32(parents), i32(tokens), i32(chosen), qkv

    def take(self, inputs):
        for mine, new in zip((self.parents, self.tokens, self.chosen, self.qkv), inputs):
            mine.copy_(new)

    def step(self):
        kv4, H, Hkv = self.kv4, self.H, self.Hkv  # noqa: F811
        kv4.pages_plan(self.page, self.lens, self.new, self.free, self.count, self.plan, self.position)
        self.tree.token_pos = self.plan.token_pos
        kv4.tree_plan(self.plan.query_start, self.parents, self.position, self.tree)
        for layer in range(self.layers):
            x = self.qkv[layer]
            kv4.qk_norm_rope(self.rope, x[:, :H], x[:, H:H + Hkv], self.tree.token_pos, self.q[layer], None, x[:, H + Hkv:],
                             self.layer_cache[layer], self.plan.slot_map)
            kv4.tree_attention(self.layer_cache[layer], self.q[layer], self.table, self.plan.seq_lens, self.scale, self.plan.query_start,
                               self.tree.tree_mask, self.nodes, self.window, self.sinks, self.out[layer], None, self.ws)
        kv4.tree_keep(self.plan.query_start, self.parents, self.tokens, self.chosen, self.lens, self.kept, self.cache, self.plan.slot_map,
                      self.layers)
        kv4.pages_trim(self.page, self.plan.seq_lens, self.lens, self.table, self.free, self.plan.free_left, self.left, self.given,
                       self.window, self.sinks)
        self.count.copy_(self.left)
        self.position.add_(self.kept.accepted)

    def state(self):
        return {"table": self.table, "free": self.free, "count": self.count, "lens": self.lens, "position": self.position,
                "path": self.kept.path, "next": self.kept.next_token, "out": self.out, "pages": self.pages}


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_generation_with_trees_and_a_window(kv4, dtype, D):  # noqa: F811
    """Steps that grow past the window.  A plain cache of all rows, in which the path is followed by hand, gives the same rows where
    anybody sees them, and attention over it the outputs; pages that were given back are full of NaN before they are used again."""
    g = Generation(kv4, dtype=dtype, D=D)
    R, n = g.R, g.nodes
    history = [[[] for _ in range(g.layers)] for _ in range(R)]     # (key, value) of the tokens kept, [Hkv, D] each
    for step in range(45):
        g.take(g.inputs(step))
        before = g.lens.tolist()
        in_use = set(g.table.cpu().numpy().reshape(-1).tolist())
        unused = torch.tensor([p for p in range(g.per_layer) if p not in in_use], device="cuda", dtype=torch.long)
        for layer in range(g.layers):
            g.pages[unused + layer * g.per_layer] = 255
        g.step()
        assert not g.plan.status.any() and not g.tree.status.any()
        parents, tokens, chosen = (t.cpu().numpy().reshape(R, n) for t in (g.parents, g.tokens, g.chosen))
        # the drafts' rows by the framework's own rotation, without a cache
        slots = g.plan.slot_map.cpu().numpy()
        for layer in range(g.layers):
            x = g.qkv[layer]
            q, k = kv4.qk_norm_rope(g.rope, x[:, :g.H], x[:, g.H:g.H + g.Hkv], g.tree.token_pos)
            assert torch.equal(q, g.q[layer])
            q, k, v = (t.float().cpu().numpy().astype(np.float64) for t in (q, k, x[:, g.H + g.Hkv:]))
            stored = [np.stack([orc.decode_rows(*orc.encode_rows(row)) for row in a]) for a in (k, v)]
            out = g.out[layer].float().cpu().numpy()
            for r in range(R):
                words = g.tree.tree_mask[r * n:(r + 1) * n].cpu().numpy().view(np.uint32)
                seen = orc.tree_seen(before[r] + n, n, words, g.window, g.sinks)
                old = history[r][layer]
                rows = [np.stack([*(o[i] for o in old), *stored[i][r * n:(r + 1) * n]]) for i in range(2)]
                for h in range(g.Hkv):
                    heads = slice(4 * h, 4 * h + 4)
                    ref, _, spread = orc.seen_attention(q[r * n:(r + 1) * n, heads], rows[0][:, h], rows[1][:, h], seen, g.scale)
                    tol = 5e-5 * spread + (np.abs(ref) * 2.0 ** -8 if dtype == torch.bfloat16 else 0)
                    assert np.all(np.abs(out[r * n:(r + 1) * n, heads] - ref) <= tol), (step, layer, r, h)
            for r in range(R):
                here, path = 0, [0]
                while True:
                    children = [c for c in range(here + 1, n) if parents[r, c] == here and tokens[r, c] == chosen[r, here]]
                    if not children:
                        break
                    here = children[0]
                    path.append(here)
                history[r][layer] += [(stored[0][r * n + i], stored[1][r * n + i]) for i in path]
                assert g.lens[r] == len(history[r][layer]) and g.kept.next_token[r] == chosen[r, here]
        # what the next token sees is where the table says, in all layers
        table, lens = g.table.cpu().numpy(), g.lens.tolist()
        for r in range(R):
            at = [t for t in range(lens[r]) if t < g.sinks or t > lens[r] - g.window]
            slots = table[r][np.array(at) // g.page] * g.page + np.array(at) % g.page
            for layer in range(g.layers):
                for i, rows in enumerate(kv4.load(g.layer_cache[layer], i32(slots), dtype=torch.float32)):
                    np.testing.assert_array_equal(rows.cpu().numpy(), np.stack([history[r][layer][t][i] for t in at]).astype(np.float32))
            gone = [j for j in range(lens[r] // g.page + 2) if all(t >= lens[r] or (t >= g.sinks and t <= lens[r] - g.window)
                                                                  for t in range(j * g.page, (j + 1) * g.page))]
            assert (table[r][gone] == -1).all()
        used = table[table >= 0].tolist()
        on_stack = g.free[:int(g.count)].tolist()
        assert sorted(used + on_stack) == list(range(g.per_layer))      # no page lost, none twice
    assert min(lens) > g.window + 20


def test_the_step_in_a_graph(kv4):  # noqa: F811
    """Captured once and replayed, with eager work and waits between, each replay against an eager twin; two graphs on one
    workspace take turns."""
    eager, graphed, other = (Generation(kv4, seed=3) for _ in range(3))
    other.ws = graphed.ws
    drafts = [eager.inputs(100 + i) for i in range(14)]
    side = torch.cuda.Stream()
    graphs = []
    for g in (eager, graphed, other):
        g.take(drafts[0])
        with torch.cuda.stream(side):
            g.step()
        side.synchronize()
    for g in (graphed, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            g.step()
        graphs.append(graph)
    for i in range(1, 14):
        for g in (eager, graphed, other):
            g.take(drafts[i])
        eager.step()
        for graph in graphs:
            graph.replay()
        if i % 3 == 0:
            torch.cuda.synchronize()
        for name, want in eager.state().items():
            assert torch.equal(graphed.state()[name], want) and torch.equal(other.state()[name], want), (i, name)
    assert int(eager.lens.min()) > 20


def test_calls_follow_their_stream(kv4):  # noqa: F811
    """Inputs that a stream is still writing when the calls are made."""
    want, g = Generation(kv4, seed=5), Generation(kv4, seed=5)
    drafts = want.inputs(7)
    want.take(drafts)
    want.step()
    side, big = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big * 1e-3
        g.take(drafts)
        g.step()
    side.synchronize()
    for name, t in want.state().items():
        assert torch.equal(g.state()[name], t), name


def test_batches_of_nothing(kv4):  # noqa: F811
    cache = kv4.Cache(torch.full((2, kv4.page_bytes(32, 2, 64)), 9, dtype=torch.uint8, device="cuda"), 32, 2, 64)
    none, empty = torch.zeros((0, 4, 64), device="cuda"), i32(np.zeros(0))
    table, lens, start = i32([[0], [1]]), i32([5, 0]), i32([0, 0, 0])
    assert kv4.window_attention(cache, none, table, lens, 0.1, 7, 0, start, 1).shape == (0, 4, 64)
    assert kv4.tree_attention(cache, none, table, lens, 0.1, start, i32(np.zeros((0, 1))), 1).shape == (0, 4, 64)
    plan = kv4.TreePlan.empty(2, 0, 5)
    kv4.tree_plan(start, empty, lens, plan)
    assert plan.status.tolist() == [0, 0]
    kept = kv4.TreeKept.empty(2, 3)
    kv4.tree_keep(start, empty, empty, empty, lens, kept, cache, empty)
    assert kept.path.tolist() == [[-1] * 3] * 2 and kept.kept_lens.tolist() == [5, 0] and kept.next_token.tolist() == [-1, -1]
    assert torch.all(cache.pages == 9)
    left, given = i32([0]), i32([7, 7])
    kv4.pages_trim(32, lens, lens, table, i32([4]), i32([1]), left, given)
    assert int(left) == 1 and given.tolist() == [0, 0] and table.tolist() == [[0], [1]]


def test_refusals(kv4):  # noqa: F811
    E = kv4.ShotKVError
    cache = kv4.Cache.empty(4, 64, 2, 128)
    q, table, lens, start = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda"), i32([[0, 1]]), i32([70]), i32([0, 3])
    mask = i32([[1], [3], [5]])
    with pytest.raises(E, match="window"):
        kv4.window_attention(cache, q, table, lens, 0.1, 0, 0, start, 3)
    with pytest.raises(E, match="unsupported"):
        kv4.window_attention(cache, q, table, lens, 0.1, None, 0, start, 3)
    with pytest.raises(E, match="n_sinks"):
        kv4.window_attention(cache, q, table, lens, 0.1, 5, -1, start, 3)
    with pytest.raises(E, match="window"):
        kv4.tree_attention(cache, q, table, lens, 0.1, start, mask, 3, -5)
    for bad, why in ((mask[:2], "shape"), (mask[:, 0], "shape"), (mask.long(), "int32"), (mask.cpu(), "GPU"), (i32(np.zeros((3, 33))), "unsupported"),
                     (i32(np.zeros((3, 0))), "unsupported"), (i32(np.zeros((3, 2)))[:, :1], "contiguous")):
        with pytest.raises(E, match=why):
            kv4.tree_attention(cache, q, table, lens, 0.1, start, bad, 3)
    with pytest.raises(E, match="workspace"):
        kv4.tree_attention(cache, q, table, lens, 0.1, start, mask, 3, workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(E, match="unsupported"):
        kv4.tree_attention(cache, q, table, lens, 0.1, None, mask)        # three tokens, one request, no starts
    ints = i32([0, 0, 0])
    with pytest.raises(E, match="unsupported"):
        kv4.tree_plan(start, ints, lens, kv4.TreePlan.empty(1, 3, 1025))
    with pytest.raises(E, match="shape"):
        kv4.tree_plan(start, ints, lens, kv4.TreePlan.empty(1, 2, 3))
    kept = kv4.TreeKept.empty(1, 3)
    with pytest.raises(E, match="slot_map"):
        kv4.tree_keep(start, ints, ints, ints, lens, kept, cache)
    with pytest.raises(E, match="unsupported"):
        kv4.tree_keep(start, ints, ints, ints, lens, kept, cache, ints, 3)        # four pages are not three layers
    with pytest.raises(E, match="unsupported"):
        kv4.tree_keep(start, ints, ints, ints, lens, kv4.TreeKept.empty(1, 0))
    with pytest.raises(E, match="shape"):
        kv4.tree_keep(start, ints, ints[:2], ints, lens, kept)
    one, given = i32([2]), i32([0])
    with pytest.raises(E, match="unsupported"):
        kv4.pages_trim(64, lens, lens, table, i32([0, 1, 2]), one, one, given)
    with pytest.raises(E, match="unsupported"):
        kv4.pages_trim(64, lens, lens, table, i32([0, 1, 2]), one, i32([0]), lens)
    with pytest.raises(E, match="window"):
        kv4.pages_trim(64, lens, lens, table, i32([0, 1, 2]), one, i32([0]), given, 0)
    with pytest.raises(E, match="unsupported"):
        kv4.pages_trim(48, lens, lens, table, i32([0, 1, 2]), one, i32([0]), given)
    torch.cuda.synchronize()
