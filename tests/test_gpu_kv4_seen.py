"""Attention over the paged 4-bit cache with windows, sinks and drafted trees, against its plain definition in 64 bits, through
the public binding.

Tolerances are those of causal attention, whose products, weights and sums these calls share: a weight is off by 2^-16 as two
bf16 numbers, a logit by some 32-bit roundings of terms whose sizes add up to less than 64 (1e-5), so an output is off by that
share of the weighted sum of |v|: 5e-5, and by its own rounding (2^-8 of it in bf16).  lse: 2e-5 + 1e-6 of its size.
"""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from test_gpu_kv4 import EDGES, TYPES, Problem, host, i32, kv4  # noqa: F401

pytestmark = pytest.mark.gpu


def random_tree(rng, n, words, kind="tree"):
    """Rows of words: ancestors in a random tree, a chain, or any bits at all, rows without one among them."""
    rows = np.zeros((n, words), dtype=np.int64)
    for i in range(n):
        if kind == "any":
            bits = rng.random(32 * words) < rng.choice([0.0, 0.2, 0.9])
            rows[i] = [int(sum(1 << b for b in range(32) if bits[32 * w + b])) for w in range(words)]
            continue
        parent = -1 if i == 0 or rng.random() < 0.1 else i - 1 if kind == "chain" else int(rng.integers(0, i))
        if parent >= 0:
            rows[i] = rows[parent]
        if i < 32 * words:
            rows[i, i // 32] |= 1 << (i % 32)
    return rows


class Seen(Problem):
    """A problem whose tokens see what `rows` (trees) or a window say."""

    def set(self, window=0, sinks=0, kind=None, words=None, seed=0):
        self.window, self.sinks, self.kind = window, sinks, kind
        if kind:
            rng = np.random.default_rng(seed)
            self.words = words or max(-(-max(max(self.news), 1) // 32), 1)
            self.rows = [random_tree(rng, n, self.words, kind) for n in self.news]
            bits = np.concatenate(self.rows) if sum(self.news) else np.zeros((0, self.words), dtype=np.int64)
            self.mask = torch.from_numpy(bits.astype(np.uint32).view(np.int32).reshape(-1, self.words)).cuda()
        return self

    def seen(self, r):
        if self.kind:
            return orc.tree_seen(self.lens[r], self.news[r], self.rows[r], self.window, self.sinks)
        return orc.window_seen(self.lens[r], self.news[r], self.window, self.sinks)

    def drop_unseen_pages(self, entry=-1):
        """Takes the pages out of the table of which no token sees a key, and fills them with bytes that read back as NaN."""
        B, table = self.cache.page_size, self.table.cpu().numpy().copy()
        dropped = 0
        for r, n in enumerate(self.lens):
            any_row = self.seen(r).any(axis=0) if self.news[r] else np.ones(n, dtype=bool)
            for j in range(-(-n // B)):
                if not any_row[j * B:(j + 1) * B].any():
                    self.cache.pages[int(table[r, j])] = 255
                    table[r, j] = entry
                    dropped += 1
        self.table = i32(table)
        return dropped

    def run(self, most=None, **kw):
        self.lse = torch.full((len(self.q), self.H), 99.0, device="cuda")
        most = max(max(self.news), 1) if most is None else most
        args = (self.cache, self.q, self.table, i32(self.lens), self.scale)
        if self.kind:
            return self.kv4.tree_attention(*args, i32(self.start), self.mask, most, self.window or None, self.sinks, None, self.lse, **kw)
        return self.kv4.window_attention(*args, self.window, self.sinks, i32(self.start), most, None, self.lse, **kw)

    def check(self, out, rows_of=None, requests=None):
        """rows_of: how many first tokens of a request were asked for."""
        out, lse, q = host(out), host(self.lse), host(self.q).astype(np.float64)
        first = np.concatenate([[0], np.cumsum(self.lens)])
        for r in range(len(self.lens)) if requests is None else requests:
            seen = self.seen(r)[:rows_of]
            mine = slice(self.start[r], self.start[r] + len(seen))
            for g in range(self.Hkv):
                heads = slice(g * self.G, (g + 1) * self.G)
                k, v = self.k[first[r]:first[r + 1], g], self.v[first[r]:first[r + 1], g]
                ref, ref_lse, spread = orc.seen_attention(q[mine, heads], k, v, seen, self.scale)
                tol = 5e-5 * spread + (np.abs(ref) * 2.0 ** -8 if self.dtype == torch.bfloat16 else 0)
                assert np.all(np.abs(out[mine, heads] - ref) <= tol + 1e-30), (r, g, np.abs(out[mine, heads] - ref).max())
                got = lse[mine, heads]
                np.testing.assert_array_equal(np.isneginf(got), np.isneginf(ref_lse), err_msg=str((r, g)))
                there = np.isfinite(ref_lse)
                assert np.all(np.abs(got[there] - ref_lse[there]) <= 2e-5 + 1e-6 * np.abs(ref_lse[there])), (r, g)


SHAPES = [(32, 8, 128, 64), (8, 1, 128, 32), (7, 1, 64, 128), (5, 5, 64, 32), (12, 2, 128, 256)]
SPANS = [(1, 0), (1, 4), (31, 1), (32, 32), (33, 31), (64, 100), (200, 33), (10**6, 7), (2**31 + 5, 2**31 + 5)]


# ---- windows and sinks -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D,page", SHAPES)
@pytest.mark.parametrize("window,sinks", SPANS)
def test_single_tokens(kv4, window, sinks, H, Hkv, D, page, dtype):  # noqa: F811
    p = Seen(kv4, EDGES, [1] * len(EDGES), H, Hkv, D, page, TYPES[dtype], seed=D + H).set(window, sinks)
    p.drop_unseen_pages()
    p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D,most", [(32, 8, 128, 2), (8, 2, 128, 4), (4, 1, 64, 8), (14, 2, 128, 3), (3, 3, 64, 16), (8, 1, 128, 5)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (33, 4), (64, 65), (300, 0)])
def test_drafts(kv4, window, sinks, H, Hkv, D, most, dtype):  # noqa: F811
    rng = np.random.default_rng(most)
    news = [most, 0, 1, most, most] + rng.integers(0, most + 1, 10).tolist()
    p = Seen(kv4, EDGES, news, H, Hkv, D, 32, TYPES[dtype], seed=most).set(window, sinks)
    p.drop_unseen_pages(10**9)
    p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D,lens,news", [
    (8, 2, 128, [300, 77, 40], [300, 20, 40]), (4, 1, 64, [515, 130], [100, 130]), (7, 1, 128, [200, 33], [65, 33]),
    (8, 8, 128, [1029], [329]), (8, 1, 64, [64, 1, 100], [64, 1, 1])])
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 70), (40, 4), (128, 1), (129, 33), (500, 64)])
def test_chunks_of_prompts(kv4, window, sinks, H, Hkv, D, lens, news, dtype):  # noqa: F811
    p = Seen(kv4, lens, news, H, Hkv, D, 64, TYPES[dtype], seed=sum(lens)).set(window, sinks)
    p.drop_unseen_pages()
    p.check(p.run())


@pytest.mark.parametrize("lens,news", [([9000, 5, 4096, 1], [1, 1, 1, 1]), ([5000, 700], [3, 2]), ([6000], [70]), ([7000, 300], [40, 16])])
@pytest.mark.parametrize("window,sinks", [(100, 4), (2500, 130)])
def test_long_caches(kv4, lens, news, window, sinks):  # noqa: F811
    p = Seen(kv4, lens, news, 8, 2, 128, 64, torch.bfloat16, seed=len(lens)).set(window, sinks)
    assert p.drop_unseen_pages() > 10
    p.check(p.run())
    q = Seen(kv4, lens, news, 4, 1, 64, 32, torch.float32, seed=len(lens)).set(window, sinks)
    q.drop_unseen_pages()
    q.check(q.run())


def test_a_window_past_every_key_is_causal_attention(kv4):  # noqa: F811
    lens, news = [300, 1000, 0, 70, 33, 2000, 90], [150, 1, 0, 5, 33, 1, 0]
    for dtype, D in ((torch.bfloat16, 128), (torch.float32, 64)):
        p = Seen(kv4, lens, news, 8, 2, D, 64, dtype, seed=D).set(2**30)
        got, lse = p.run(), p.lse
        p.check(got)
        if dtype == torch.float32:      # (chunks in bf16 have kernels of their own, whose sums are of other parts)
            want = Problem.run(p)
            assert torch.equal(got, want) and torch.equal(lse, p.lse)


def test_mixed_batches_with_a_window(kv4):  # noqa: F811
    """Chunks, drafts and single tokens in one call, over tables wide enough for two kernels and not."""
    lens, news = [300, 1000, 0, 70, 33, 2000, 90, 512], [150, 1, 0, 8, 33, 1, 0, 9]
    for dtype, D in ((torch.bfloat16, 128), (torch.float32, 64)):
        for wide in (0, 4000):
            p = Seen(kv4, lens, news, 8, 2, D, 64, dtype, seed=D).set(150, 5)
            if wide:
                p.table = torch.cat([p.table, torch.full((len(lens), wide), -1, dtype=torch.int32, device="cuda")], dim=1)
            p.check(p.run())


def test_many_requests_with_a_window(kv4):  # noqa: F811
    rng = np.random.default_rng(0)
    p = Seen(kv4, rng.integers(0, 190, 700), [1] * 700, 4, 2, 64, 32, torch.bfloat16).set(40, 3)
    p.drop_unseen_pages()
    p.check(p.run())
    news = np.where(np.arange(150) % 3 == 0, 40, 9)
    p = Seen(kv4, rng.integers(45, 250, 150), news.tolist(), 4, 2, 64, 32, torch.bfloat16).set(40, 3)
    p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("requests,most", [(5, 1), (70, 1), (140, 3), (130, 16)])
def test_few_blocks_of_many_requests(kv4, requests, most, dtype):  # noqa: F811
    """Windows and short tables of up to 16 blocks and of up to 36, with as many requests as there are CUs and fewer."""
    rng = np.random.default_rng(requests)
    news = rng.integers(0, most + 1, requests)
    news[::3] = most
    lens = rng.integers(0, 1100, requests)
    lens[:3] = 0, 1100, 512
    for window, sinks in ((300, 4), (700, 40)):
        p = Seen(kv4, lens, news.tolist(), 4, 2, 64, 32, TYPES[dtype], seed=most).set(window, sinks)
        p.drop_unseen_pages()
        p.check(p.run())
        p.set(window, sinks, "tree", seed=most)
        p.check(p.run())
    p = Seen(kv4, np.minimum(lens, 400), news.tolist(), 4, 2, 64, 32, TYPES[dtype], seed=most).set(kind="any", seed=most)
    p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D", [(8, 2, 128), (4, 2, 64), (5, 1, 128)])
@pytest.mark.parametrize("requests,most", [(1, 300), (9, 70), (40, 33), (70, 20)])
def test_tiles_of_requests_as_long(kv4, requests, most, H, Hkv, D, dtype):  # noqa: F811
    """Requests of (nearly) as many new tokens, whose tiles need not be cut: a few of fewer, of none and of more than are taken."""
    rng = np.random.default_rng(requests)
    news, lens = np.full(requests, most), rng.integers(most, 700, requests)
    if requests > 8:
        news[[0, 3, 5]], lens[[1, 5]] = (3, 0, most + 9), (0, most + 9)
    for window, sinks, kind in ((150, 4, None), (1, 0, None), (0, 0, "tree"), (90, 33, "any")):
        p = Seen(kv4, lens, news.tolist(), H, Hkv, D, 32, TYPES[dtype], seed=most).set(window, sinks, kind, seed=most)
        if not kind:
            p.drop_unseen_pages()
        out = p.run(most)
        p.check(out, requests=[r for r in range(requests) if news[r] <= most])
        for r in np.flatnonzero(news > most):
            p.check(out, rows_of=most, requests=[r])
            assert not out[p.start[r] + most:p.start[r + 1]].any()


@pytest.mark.parametrize("news", [[1], [4], [9], [40]])
def test_what_a_window_leaves_out_does_not_reach_a_row(kv4, news):  # noqa: F811
    """Keys and values that are not finite: before the window in the block where it begins, between sinks, behind a token."""
    for D, dtype in ((128, torch.bfloat16), (64, torch.float32)):
        def values(k, v):
            for at in (3, 20, 60, 99):
                k[at], v[at, :, 40:] = np.nan, np.inf
        # the first token is at 200 - n and sees 200 - n - 99 on: past 99 for all
        p = Seen(kv4, [200], news, 4, 2, D, 32, dtype, values=values).set(100 - news[0] + 1, 3)
        p.check(p.run())
        p.set(100, 3 + 1)       # token 3 is a sink
        assert np.isnan(host(p.run())).all() and np.isnan(host(p.lse)).all()

        def only_values(k, v):
            v[3, :, 40:] = np.inf
            v[60, :, :32] = np.inf
        p = Seen(kv4, [200], news, 4, 2, D, 32, dtype, values=only_values).set(100 - news[0] + 1, 4)
        out = host(p.run())
        assert np.isfinite(out[:, :, :32]).all() and np.isnan(out[:, :, 32:]).all() and np.isfinite(host(p.lse)).all()


def test_a_request_cut_by_max_q_len_keeps_its_window(kv4):  # noqa: F811
    for H, Hkv, most in ((8, 2, 3), (8, 2, 20), (4, 4, 50)):
        p = Seen(kv4, [500], [70], H, Hkv, 128, 64, torch.bfloat16).set(90, 3)
        out = p.run(most)
        p.check(out, rows_of=most)
        assert not out[most:].any() and torch.all(p.lse[most:] == 99)


# ---- trees -----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["tree", "chain", "any"])
@pytest.mark.parametrize("H,Hkv,D,most", [(32, 8, 128, 8), (8, 2, 128, 4), (4, 1, 64, 2), (14, 2, 128, 16), (3, 3, 64, 33), (8, 1, 128, 20),
                                          (8, 8, 128, 64), (10, 2, 64, 70)])
def test_trees(kv4, H, Hkv, D, most, kind, dtype):  # noqa: F811
    """Drafts of all numbers, fewer in the cache than there are among them (rows that see nothing), and none."""
    rng = np.random.default_rng(most)
    news = [most, 0, 1, most, most] + rng.integers(0, most + 1, 10).tolist()
    p = Seen(kv4, EDGES, news, H, Hkv, D, 32, TYPES[dtype], seed=most).set(kind=kind, seed=most)
    out = p.run()
    p.check(out)
    assert np.isneginf(host(p.lse)[:most]).all() and not host(out)[:most].any()     # a request without a token in the cache


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D,most", [(8, 2, 128, 8), (4, 1, 64, 5), (8, 1, 128, 30), (4, 4, 64, 70)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 2), (64, 40), (150, 4), (10**6, 3)])
def test_trees_with_a_window(kv4, window, sinks, H, Hkv, D, most, dtype):  # noqa: F811
    rng = np.random.default_rng(most)
    news = [most, 0, 1, most, most] + rng.integers(0, most + 1, 10).tolist()
    for kind in ("tree", "any"):
        p = Seen(kv4, EDGES, news, H, Hkv, D, 32, TYPES[dtype], seed=most).set(window, sinks, kind, seed=most)
        p.drop_unseen_pages()
        p.check(p.run())


@pytest.mark.parametrize("lens,news", [([9000, 5, 4096, 31], [7, 5, 8, 31]), ([5000, 700], [26, 64]), ([6000], [130]), ([3277], [26])])
def test_trees_over_long_caches(kv4, lens, news):  # noqa: F811
    for kind, window in (("tree", 0), ("any", 2500)):
        p = Seen(kv4, lens, news, 8, 2, 128, 64, torch.bfloat16, seed=len(lens)).set(window, 4, kind)
        p.drop_unseen_pages()
        p.check(p.run())
        q = Seen(kv4, lens, news, 4, 1, 64, 32, torch.float32, seed=len(lens)).set(window, 4, kind)
        q.check(q.run())


def test_more_and_fewer_words_than_drafts(kv4):  # noqa: F811
    """Bits of drafts that a request does not have, and drafts that have no bits."""
    for news, words in (([7, 20], 3), ([70, 40], 2), ([70, 40], 1), ([7, 3], 32)):
        p = Seen(kv4, [300, 45], news, 8, 2, 128, 32, torch.bfloat16, seed=words).set(kind="any", words=words)
        p.check(p.run())
        p.set(33, 2, "any", words=words)
        p.check(p.run())


def test_a_lower_triangle_is_causal_attention(kv4):  # noqa: F811
    for news in ([5, 8, 1], [40, 33, 64]):
        for dtype in TYPES.values():
            p = Seen(kv4, [300, 77, 64], news, 8, 2, 128, 64, dtype).set(kind="tree")
            p.rows = [np.array([[((1 << (i + 1)) - 1 >> 32 * w) & (2**32 - 1) for w in range(p.words)] for i in range(n)]) for n in news]
            p.mask = torch.from_numpy(np.concatenate(p.rows).astype(np.uint32).view(np.int32)).cuda()
            # (the sums are of other parts than those of causal attention, which cuts its work elsewhere: no bits to compare)
            assert all(np.array_equal(p.seen(r), orc.window_seen(p.lens[r], n, 2**30, 0)) for r, n in enumerate(news))
            p.check(p.run())


@pytest.mark.parametrize("n", [4, 8, 12, 40])
def test_drafts_of_other_branches_do_not_reach_a_row(kv4, n):  # noqa: F811
    """A draft whose keys and values are not finite: rows that see it are NaN, all others what they are without it."""
    for D, dtype in ((128, torch.bfloat16), (64, torch.float32)):
        for keys in (True, False):
            def values(k, v):
                if keys:
                    k[100 + 1] = np.nan
                v[100 + 1, :, 40:] = np.inf
            p = Seen(kv4, [100 + n], [n], 4, 2, D, 32, dtype, values=values).set(kind="tree", seed=n)
            out, lse = host(p.run()), host(p.lse)
            sees = p.seen(0)[:, 101]
            assert sees.any() and not sees.all()
            assert np.isnan(out[sees][:, :, 32:]).all() and np.isfinite(out[~sees]).all()
            assert np.isnan(out[sees]).all() if keys else np.isfinite(out[sees][:, :, :32]).all()
            assert np.isnan(lse[sees]).all() if keys else np.isfinite(lse).all()
            q = host(p.q).astype(np.float64)
            for g in range(2):
                k, v = (np.nan_to_num(a[:, g], posinf=0.0) for a in (p.k, p.v))
                ref, _, spread = orc.seen_attention(q[:, 2 * g:2 * g + 2], k, v, p.seen(0), p.scale)
                off = np.abs(out[:, 2 * g:2 * g + 2] - ref)[~sees]
                assert np.all(off <= (5e-5 * spread + (np.abs(ref) * 2.0 ** -8 if dtype == torch.bfloat16 else 0))[~sees])


def test_a_tree_cut_by_max_q_len_sees_among_all(kv4):  # noqa: F811
    for H, Hkv, n, most in ((8, 2, 20, 3), (8, 2, 70, 20), (4, 4, 70, 50)):
        for window in (0, 50):
            p = Seen(kv4, [300], [n], H, Hkv, 128, 64, torch.bfloat16).set(window, 3, "any")
            out = p.run(most)
            p.check(out, rows_of=most)
            assert not out[most:].any() and torch.all(p.lse[most:] == 99)


def test_a_tree_of_one_without_starts(kv4):  # noqa: F811
    """query_start None: a token per request, that sees itself if its bit is set."""
    p = Seen(kv4, [70, 1, 300], [1, 1, 1], 8, 2, 128, 64, torch.bfloat16).set(kind="tree")
    p.rows = [np.array([[1]]), np.array([[0]]), np.array([[-2 & 0xffffffff]])]
    p.mask = i32([[1], [0], [-2]])
    want = p.run()
    p.check(want)
    assert not want[1].any()
    assert torch.equal(kv4.tree_attention(p.cache, p.q, p.table, i32(p.lens), p.scale, None, p.mask), want)


def test_rows_past_the_requests_stay(kv4):  # noqa: F811
    """Starts that do not begin at 0 and end before the batch does: other rows are left as they were."""
    for news in ([3, 4], [40, 30]):
        p = Seen(kv4, [100, 90], news, 8, 2, 128, 64, torch.bfloat16).set(kind="tree")
        want, T = p.run(), sum(news)
        pad = lambda t: torch.cat([t[:2], t, t[:3]]).contiguous()  # noqa: E731
        for window in (0, 10**6):
            out, lse = torch.full((T + 5, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((T + 5, 8), 5.0, device="cuda")
            if window:
                kv4.window_attention(p.cache, pad(p.q), p.table, i32(p.lens), p.scale, window, 0, i32(p.start + 2), max(news), out, lse)
            else:
                kv4.tree_attention(p.cache, pad(p.q), p.table, i32(p.lens), p.scale, i32(p.start + 2), pad(p.mask), max(news), None, 0, out, lse)
                assert torch.equal(out[2:2 + T], want)
            for x in (out, lse):
                assert torch.all(x[:2] == 5) and torch.all(x[2 + T:] == 5) and not torch.all(x[2:2 + T] == 5)


def test_rows_of_any_layout(kv4):  # noqa: F811
    for kind, window in (("tree", 0), (None, 40)):
        p = Seen(kv4, [70, 300], [2, 2], 8, 2, 128, 64, torch.bfloat16).set(window, 3, kind)
        want = p.run()
        wide = torch.zeros((4, 12, 128), dtype=torch.bfloat16, device="cuda")
        wide[:, 2:10] = p.q
        out = torch.zeros((8, 4, 128), dtype=torch.bfloat16, device="cuda")
        args = (p.cache, wide[:, 2:10], p.table, i32(p.lens), p.scale)
        if kind:
            kv4.tree_attention(*args, i32(p.start), p.mask, 2, out=out.transpose(0, 1))
        else:
            kv4.window_attention(*args, 40, 3, i32(p.start), 2, out.transpose(0, 1))
        assert torch.equal(out.transpose(0, 1), want)


def test_results_repeat_whatever_the_workspace_held(kv4):  # noqa: F811
    for news, kind in (([1, 1, 1], None), ([16, 3, 9], "tree"), ([64, 40, 50], "tree"), ([300, 70, 64], None)):
        p = Seen(kv4, [4000, 700, 64], news, 32, 8, 128, 64, torch.bfloat16).set(900, 4, kind)
        most = max(news)
        ws = kv4.tree_attention_workspace(p.cache, p.q, p.table, most, 900, 4) if kind else \
            kv4.window_attention_workspace(p.cache, p.q, p.table, 900, 4, most)
        first, lse = p.run(workspace=ws).clone(), p.lse.clone()
        ws.fill_(255)
        assert torch.equal(p.run(workspace=ws), first) and torch.equal(p.lse, lse)


def test_a_workspace_of_the_largest_call_serves_others(kv4):  # noqa: F811
    """Fewer requests, shorter windows and fewer tokens, one after the other on one workspace, each in a launch of its own kind."""
    for kind in (None, "tree"):
        large = Seen(kv4, [3000] * 40, [16] * 40, 32, 8, 64, 64, torch.bfloat16).set(2500, 4, kind)
        ws = kv4.tree_attention_workspace(large.cache, large.q, large.table, 16, 2500, 4) if kind else \
            kv4.window_attention_workspace(large.cache, large.q, large.table, 2500, 4, 16)
        for lens, news, window in (([3000, 50], [1, 1], 2500), ([3000, 7, 700], [4, 0, 8], 300), ([2900] * 34, [1] * 34, 900), ([300], [16], 2500)):
            p = Seen(kv4, lens, news, 32, 8, 64, 64, torch.bfloat16, seed=window).set(window, 4, kind)
            ws.fill_(255)
            p.check(p.run(workspace=ws))


def test_calls_on_two_streams_at_once(kv4):  # noqa: F811
    """Each with a workspace of its own, over one cache, again and again."""
    for news, kind in (([1, 1, 1], None), ([20, 3, 9], "tree"), ([200, 70, 64], None)):
        p = Seen(kv4, [4000, 700, 200], news, 32, 8, 128, 64, torch.bfloat16).set(900, 4, kind)
        want, lse = p.run(), p.lse
        p.check(want)
        starts, lens = i32(p.start), i32(p.lens)
        calls = []
        for _ in range(2):
            ws = kv4.tree_attention_workspace(p.cache, p.q, p.table, max(news), 900, 4) if kind else \
                kv4.window_attention_workspace(p.cache, p.q, p.table, 900, 4, max(news))
            calls.append((torch.cuda.Stream(), torch.zeros_like(p.q), torch.zeros_like(lse), ws))
        torch.cuda.synchronize()
        for _ in range(20):
            for stream, out, own, ws in calls:
                with torch.cuda.stream(stream):
                    if kind:
                        kv4.tree_attention(p.cache, p.q, p.table, lens, p.scale, starts, p.mask, max(news), 900, 4, out, own, ws)
                    else:
                        kv4.window_attention(p.cache, p.q, p.table, lens, p.scale, 900, 4, starts, max(news), out, own, ws)
        torch.cuda.synchronize()
        for _, out, own, _ in calls:
            assert torch.equal(out, want) and torch.equal(own, lse)


def test_requests_that_share_their_first_pages(kv4):  # noqa: F811
    """The pages of a common prompt in several rows of the table, and one request in two of them."""
    for news, kind, window in (([1, 1, 1], None, 300), ([6, 6, 6], "tree", 0), ([40, 40, 40], "tree", 300)):
        p = Seen(kv4, [640, 640, 640], news, 8, 2, 128, 64, torch.bfloat16, seed=news[0]).set(window, 70, kind)
        table = p.table.clone()
        table[1, :5] = table[0, :5]
        table[2] = table[0]
        p.table = table
        for a in (p.k, p.v):
            a[640:960], a[1280:] = a[:320], a[:640]
        p.check(p.run())


def test_peaked_rows_and_sinks_far_ahead(kv4):  # noqa: F811
    """A sink whose logits are far above all others, and far below."""
    for factor in (30.0, -30.0):
        def values(k, v):
            k[:4] *= factor
        p = Seen(kv4, [1000, 40], [1, 1], 8, 2, 128, 64, torch.float32, values=values, spread=0.2).set(100, 4)
        p.check(p.run())
        p = Seen(kv4, [1000, 80], [40, 33], 8, 2, 128, 64, torch.bfloat16, values=values, spread=0.2).set(100, 4)
        p.check(p.run())


def test_a_pool_of_more_than_4_gib(kv4):  # noqa: F811
    """Offsets past 32 bits: a request whose last pages lie at the end of a pool of 5 GiB."""
    D, H, page = 128, 8, 128
    n_pages = 5 * 2**30 // kv4.page_bytes(page, H, D)
    cache = kv4.Cache.empty(n_pages, page, H, D)
    table = i32([[n_pages - 1, -1, n_pages - 3]])
    slots = np.concatenate([(n_pages - 1) * page + np.arange(128), np.full(128, -1), (n_pages - 3) * page + np.arange(44)])
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = torch.randn((2, 300, H, D), generator=g, device="cuda")
    kv4.store(cache, k, v, i32(slots))
    kk, vv = (host(t).astype(np.float64) for t in kv4.load(cache, i32(slots), dtype=torch.float32))
    q = torch.randn((40, H, D), generator=g, device="cuda")
    for n in (1, 40):
        out = host(kv4.window_attention(cache, q[:n].contiguous(), table, i32([300]), 0.1, 3, 30, i32([0, n]), n))
        seen = orc.window_seen(300, n, 3, 30)
        for h in range(H):
            ref, _, s = orc.seen_attention(host(q)[:n, h:h + 1], kk[:, h], vv[:, h], seen, 0.1)
            assert np.all(np.abs(out[:, h:h + 1] - ref) <= 5e-5 * s)
