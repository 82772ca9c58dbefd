"""Pins of the plain definitions of windows, sinks, drafted trees and pages that go back: values worked out by hand, and
attention against torch's own with the mask spelled out."""
import math

import numpy as np
import torch

from oracle import kv4_oracle as orc


def test_windows_by_hand():
    seen = orc.window_seen(7, 2, 3, 0)
    assert seen.astype(int).tolist() == [[0, 0, 0, 1, 1, 1, 0], [0, 0, 0, 0, 1, 1, 1]]
    seen = orc.window_seen(7, 2, 1, 2)
    assert seen.astype(int).tolist() == [[1, 1, 0, 0, 0, 1, 0], [1, 1, 0, 0, 0, 0, 1]]
    # sinks that a token's own position has not reached are not seen, nor anything by a token that is not cached
    assert orc.window_seen(3, 3, 1, 3).astype(int).tolist() == [[1, 0, 0], [1, 1, 0], [1, 1, 1]]
    assert orc.window_seen(1, 3, 4, 4).astype(int).tolist() == [[0], [0], [1]]
    for n_keys, n_new in ((9, 4), (33, 33), (2, 5)):
        causal = np.arange(n_keys)[None] <= n_keys - n_new + np.arange(n_new)[:, None]
        np.testing.assert_array_equal(orc.window_seen(n_keys, n_new, 100, 0), causal)


def test_trees_by_hand():
    words = [[0b001], [0b011], [0b101]]
    assert orc.tree_seen(5, 3, words).astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 1, 0, 1]]
    # a window of 2: the first draft is at position 2 and sees 1 on, its children are both at 3
    assert orc.tree_seen(5, 3, words, 2, 0).astype(int).tolist() == [[0, 1, 1, 0, 0], [0, 0, 1, 1, 0], [0, 0, 1, 0, 1]]
    assert orc.tree_seen(5, 3, words, 2, 1).astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 0, 1, 1, 0], [1, 0, 1, 0, 1]]
    # bits that no draft has, and a row without any: at the position before the drafts
    assert orc.tree_seen(4, 2, [[0b1100], [0b0110]], 1, 0).astype(int).tolist() == [[0, 1, 0, 0], [0, 0, 0, 1]]
    # two of the three drafts are cached
    assert orc.tree_seen(2, 3, [[0b001], [0b011], [0b101]]).astype(int).tolist() == [[0, 0], [1, 0], [0, 1]]


def test_attention_over_what_is_seen():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((5, 3, 64)), rng.standard_normal((20, 64)), rng.standard_normal((20, 64))
    seen = rng.random((5, 20)) < 0.4
    seen[2] = False
    out, lse, spread = orc.seen_attention(q, k, v, seen, 0.3)
    t = lambda a: torch.from_numpy(a)  # noqa: E731
    z = (t(q) @ t(k).T * 0.3).masked_fill(~t(seen)[:, None], -math.inf)
    np.testing.assert_allclose(lse, torch.logsumexp(z, -1).numpy(), atol=1e-13)
    w = torch.softmax(z, -1).nan_to_num(0.0)
    np.testing.assert_allclose(out, (w @ t(v)).numpy(), atol=1e-13)
    np.testing.assert_allclose(spread, (w @ t(v).abs()).numpy(), atol=1e-13)
    assert not out[2].any() and np.isneginf(lse[2]).all()
    causal = orc.attention(q, k, v, 5, 0.3)
    for a, b in zip(causal, orc.seen_attention(q, k, v, orc.window_seen(20, 5, 20, 0), 0.3)):
        np.testing.assert_array_equal(a, b)


def test_tree_plan_by_hand():
    #        0        0
    #       1 2      33 is the last of a chain of 34
    #      3
    parents = [-1, 0, 0, 1] + list(range(-1, 33)) + [-1, 1]
    mask, pos, status = orc.tree_plan([0, 4, 38, 40, 40], parents, [10, 5, 0, 7], 2)
    assert mask[:4].tolist() == [[1, 0], [3, 0], [5, 0], [11, 0]] and pos[:4].tolist() == [10, 11, 11, 12]
    assert mask[37].tolist() == [2**32 - 1, 3] and pos[37] == 38
    assert status.tolist() == [0, 0, -6, 0] and not mask[38:].any() and (pos[38:] == -1).all()     # token 1 names itself
    assert orc.tree_plan([0, 4, 38], parents, [10, 5], 1)[2].tolist() == [0, -5]


def test_tree_keep_by_hand():
    #  0 -> 1 (7), 2 (8), 3 (8);  2 -> 4 (9);  3 -> 5 (9);  4 -> 6 (1)
    parents, tokens = [-1, 0, 0, 0, 2, 3, 4], [3, 7, 8, 8, 9, 9, 1]
    chosen = [8, 0, 9, 9, 4, 4, 4]
    slots = np.arange(100, 107)
    path, accepted, following, lens, moves = orc.tree_keep([0, 7], parents, tokens, chosen, [50], 5, slots, 200)
    assert path.tolist() == [[0, 2, 4, -1, -1]] and accepted.tolist() == [3] and following.tolist() == [4] and lens.tolist() == [53]
    assert moves == [(102, 101), (104, 102)]
    assert orc.tree_keep([0, 7], parents, tokens, chosen, [50], 2)[0].tolist() == [[0, 2]]
    assert orc.tree_keep([0, 7], parents, tokens, [-1] * 7, [50], 5)[1:3] == (np.array([1]), np.array([-1]))
    slots[0] = -1
    path, accepted, following, lens, moves = orc.tree_keep([0, 7], parents, tokens, chosen, [50], 5, slots, 200)
    assert (path == -1).all() and accepted.tolist() == [0] and following.tolist() == [-1] and lens.tolist() == [50] and not moves


def test_a_moved_row_is_the_stored_one():
    rng = np.random.default_rng(2)
    for D in (64, 128):
        pool = rng.integers(0, 256, 2 * orc.page_bytes(32, 2, D)).astype(np.uint8)
        k, v = rng.standard_normal((2, 2, D))
        want = pool.copy()
        orc.store(pool, 32, 2, D, 45, k, v)
        orc.store(want, 32, 2, D, 45, k, v)
        orc.store(want, 32, 2, D, 7, k, v)
        orc.move(pool, 32, 2, D, 45, 7)
        np.testing.assert_array_equal(pool, want)


def test_trim_by_hand():
    table = np.array([[10, 11, 12, 13, 14], [20, -1, 22, 23, 24]])
    stack = np.array([1, 2, 0, 0, 0, 0, 0])
    # 130 tokens of 160 stay: the last page goes; the second request has 100 of 70 cached ones and keeps all
    out, free, left, given = orc.pages_trim(32, [160, 70], [128, 100], table, stack, 2)
    assert out.tolist() == [[10, 11, 12, 13, -1], [20, -1, 22, 23, 24]] and free.tolist() == [1, 2, 14, 0, 0, 0, 0]
    assert left == 3 and given.tolist() == [1, 0]
    # the next token is number 160 and sees 96 on: pages 1 and 2 hold tokens 32 to 95; page 0 has sinks
    out, free, left, given = orc.pages_trim(32, [160, 160], [160, 159], table, stack, 2, 65, 4)
    assert out.tolist() == [[10, -1, -1, 13, 14], [20, -1, 22, 23, 24]]
    assert free.tolist() == [1, 2, 12, 11, 0, 0, 0] and left == 4 and given.tolist() == [2, 0]
    # without sinks the first page goes too; a stack without room drops what would pass it
    out, free, left, given = orc.pages_trim(32, [160, 0], [160, 0], table, stack[:3], 2, 65, 0)
    assert out[0].tolist() == [-1, -1, -1, 13, 14] and free.tolist() == [1, 2, 12] and left == 3 and given.tolist() == [3, 0]
