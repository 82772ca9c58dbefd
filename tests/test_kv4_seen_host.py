"""What the entry points for windows, trees and pages that go back say without a GPU: every call here ends at its checks, before
any pointer is read or any work enqueued."""
import ctypes
import os

import pytest
import torch

OK, NULL, SHAPE, WORKSPACE, ALIGN = 0, -1, -2, -3, -4
SOME, ODD = 4096, 4100      # pointers that nobody reads


@pytest.fixture(scope="module")
def kv4():
    from paper_2502_01941_amd import build, kv4, shotkv
    if not os.path.exists(shotkv.LIB_PATH):
        build.build(force=True)
    kv4.load_library()
    return kv4


def config(kv4, heads=8, kv_heads=2, D=128, scale=1.0):
    return kv4._heads(heads, kv_heads, D, torch.bfloat16, scale)


def cache(kv4, pages=SOME, n_pages=8, page_size=64):
    return kv4._Cache(pages, n_pages, page_size)


def rows(kv4, data=SOME, stride=1024):
    return kv4._Rows(data, 0, stride, 128, 100)


def attend(kv4, what, cfg=None, R=2, T=9, most=5, pool=0, table=SOME, max_pages=4, lens=SOME, start=SOME, mask=SOME, words=1, window=3, sinks=0,
           q=0, out=0, ws=SOME, ws_bytes=0):
    lib, cfg = kv4.load_library(), cfg or config(kv4)
    pool, q, out = (cache(kv4) if pool == 0 else pool), (rows(kv4) if q == 0 else q), (rows(kv4) if out == 0 else out)
    tree = (mask, words) if what == "tree" else ()
    return getattr(lib, f"shotkv_kv4_{what}_attention")(cfg, R, T, most, pool, table, max_pages, lens, start, *tree, window, sinks, q, out, None, ws,
                                                        ws_bytes, None)


def workspace(kv4, what, cfg=None, R=2, T=9, most=5, page=64, max_pages=4, window=3, sinks=0):
    return getattr(kv4.load_library(), f"shotkv_kv4_{what}_attention_workspace_bytes")(cfg or config(kv4), R, T, most, page, max_pages, window, sinks)


@pytest.mark.parametrize("what", ["window", "tree"])
def test_attention(kv4, what):
    # whatever else is right, the workspace of no bytes is too small: nothing is ever launched
    assert attend(kv4, what) == WORKSPACE
    assert attend(kv4, what, pool=None) == NULL and attend(kv4, what, pool=cache(kv4, None)) == NULL
    for name in ("table", "lens", "ws", "q", "out"):
        assert attend(kv4, what, **{name: None}) == NULL, name
    assert attend(kv4, what, q=rows(kv4, None)) == NULL
    for wrong in (dict(R=0), dict(R=65536, T=65536), dict(T=-1), dict(T=2**28 + 1), dict(most=0), dict(max_pages=0), dict(max_pages=2**24 + 1),
                  dict(sinks=-1), dict(window=-1), dict(window=-2**31), dict(cfg=config(kv4, 12, 1)), dict(cfg=config(kv4, D=96)),
                  dict(cfg=config(kv4, scale=0.0)), dict(pool=cache(kv4, page_size=48)), dict(pool=cache(kv4, n_pages=0)), dict(start=None)):
        assert attend(kv4, what, **wrong) == SHAPE, wrong
    assert attend(kv4, what, window=0) == (SHAPE if what == "window" else WORKSPACE)
    for odd in (dict(q=rows(kv4, ODD)), dict(out=rows(kv4, stride=1001)), dict(pool=cache(kv4, ODD)), dict(ws=ODD)):
        assert attend(kv4, what, **odd) == ALIGN, odd
    assert attend(kv4, what, T=0, q=None, out=None, mask=None) == OK      # no tokens, and there need be no rows


def test_masks(kv4):
    assert attend(kv4, "tree", mask=None) == NULL
    assert attend(kv4, "tree", words=0) == SHAPE and attend(kv4, "tree", words=33) == SHAPE and attend(kv4, "tree", words=32) == WORKSPACE


@pytest.mark.parametrize("what", ["window", "tree"])
def test_workspaces(kv4, what):
    """Something for every shape that a call takes, nothing for others, and no more with a window than without."""
    least = workspace(kv4, what)
    assert least > 0
    for most in (1, 2, 8, 9, 64, 2048):
        for heads, kv_heads in ((64, 8), (8, 8), (5, 1)):
            cfg = config(kv4, heads, kv_heads)
            shapes = [workspace(kv4, what, cfg, 4, 4 * most, most, 64, 4096, window, sinks) for window, sinks in
                      ((1, 0), (1000, 4), (2**30, 0), (2**31 - 1, 2**31 - 1))]
            assert 0 < shapes[0] <= shapes[1] <= shapes[2] == shapes[3]
    assert workspace(kv4, what, window=-1) == 0 and workspace(kv4, what, sinks=-1) == 0 and workspace(kv4, what, page=48) == 0
    assert workspace(kv4, what, window=0) == (0 if what == "window" else workspace(kv4, what, window=2**30))
    assert workspace(kv4, what, None, 65535, 65535, 1) > 0 and workspace(kv4, what, None, 65536, 65536, 1) == 0
    assert workspace(kv4, what, None, 1, 1, 1, 32, 2**25) > 0 and workspace(kv4, what, None, 1, 1, 1, 32, 2**25 + 1) == 0


@pytest.mark.parametrize("what", ["window", "tree"])
@pytest.mark.parametrize("most", [1, 3, 8, 200])
def test_a_workspace_serves_smaller_calls(kv4, what, most):
    """Fewer requests, shorter windows and narrower tables never need more: one workspace for the largest call does."""
    cfg = config(kv4, 32, 8)
    grows = [[workspace(kv4, what, cfg, R, R * most, most, 64, 512, 300) for R in (1, 2, 31, 32, 33, 64, 300, 65535)],
             [workspace(kv4, what, cfg, 40, 40 * most, most, 64, 512, w) for w in (1, 60, 300, 700, 1000, 1100, 1500, 9000, 2**30)],
             [workspace(kv4, what, cfg, 40, 40 * most, most, 64, pages, 2**30) for pages in (1, 7, 8, 9, 17, 18, 19, 100, 4000)]]
    for sizes in grows:
        assert sizes[0] > 0 and sizes == sorted(sizes), sizes


def test_tree_plan(kv4):
    call = kv4.load_library().shotkv_tree_plan
    for wrong in ((0, 5, 1), (65536, 5, 1), (1, -1, 1), (1, 2**28 + 1, 1), (1, 5, 0), (1, 5, 33)):
        assert call(wrong[0], wrong[1], SOME, SOME, SOME, wrong[2], SOME, SOME, SOME, None) == SHAPE
    for i in (2, 3, 4, 6, 7, 8):
        args = [1, 5, SOME, SOME, SOME, 1, SOME, SOME, SOME, None]
        args[i] = None
        assert call(*args) == NULL


def test_tree_keep(kv4):
    call = kv4.load_library().shotkv_tree_keep
    good = [2, 9, SOME, SOME, SOME, SOME, SOME, 4, SOME, SOME, SOME, SOME, cache(kv4), 2, 128, 1, SOME, None]

    def but(*changes):
        args = list(good)
        for i, x in changes:
            args[i] = x
        return call(*args)
    for i, bad in ((0, 0), (0, 65536), (1, -1), (1, 2**28 + 1), (7, 0), (7, 2**28 + 1), (13, 0), (13, 65), (14, 96), (15, 0), (15, -1), (15, 3),
                   (12, cache(kv4, page_size=48))):
        assert but((i, bad)) == SHAPE, (i, bad)
    assert but((12, cache(kv4, n_pages=2**17)), (13, 64), (15, 2**13)) == SHAPE       # more pairs of layer and head than a grid has
    for i in (2, 3, 4, 5, 6, 8, 9, 10, 11, 16):
        assert but((i, None)) == NULL, i
    assert but((12, cache(kv4, None))) == NULL and but((12, cache(kv4, ODD))) == ALIGN


def test_trim(kv4):
    call = kv4.load_library().shotkv_pages_trim
    good = [2, 64, 4, SOME, SOME + 64, 0, 0, SOME + 128, SOME + 256, 8, SOME + 512, SOME + 520, SOME + 640, None]

    def but(*changes):
        args = list(good)
        for i, x in changes:
            args[i] = x
        return call(*args)
    for i, bad in ((0, 0), (0, 65536), (1, 48), (1, 0), (2, 0), (2, 2**24 + 1), (5, -1), (6, -1), (9, -1), (11, SOME + 512), (12, SOME), (12, SOME + 64)):
        assert but((i, bad)) == SHAPE, (i, bad)
    # arrays that are written and are another argument as well
    for i, others in ((11, (3, 4, 7, 8, 10, 12)), (12, (3, 4, 7, 8, 10)), (8, (7,))):
        for j in others:
            assert but((i, good[j])) == SHAPE, (i, j)
    for i in (3, 4, 7, 8, 10, 11, 12):
        assert but((i, None)) == NULL, i


def test_the_binding_takes_windows_of_any_size(kv4):
    """Whole numbers past 32 bits are not cut to their low bits."""
    assert kv4._window(None, 0) == (0, 0) and kv4._window(7, 3) == (7, 3)
    assert kv4._window(2**32 + 5, 2**33) == (2**30, 2**30)
    for bad in ((0, 0), (-1, 0), (5, -1)):
        with pytest.raises(kv4.ShotKVError):
            kv4._window(*bad)
