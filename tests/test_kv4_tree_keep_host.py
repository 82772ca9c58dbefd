"""What the call that keeps the drafts of a plan says without a GPU: every call here ends at its checks."""
import pytest

from test_kv4_seen_host import ALIGN, NULL, ODD, SHAPE, SOME, cache, kv4  # noqa: F401  (kv4 is the fixture)


def test_tree_keep_planned(kv4):  # noqa: F811
    call = kv4.load_library().shotkv_tree_keep_planned
    good = [2, 9, SOME, SOME, SOME, SOME, SOME, 4, SOME, SOME, SOME, SOME, cache(kv4), 2, 128, 1, SOME, SOME + 128, None]

    def but(*changes):
        args = list(good)
        for i, x in changes:
            args[i] = x
        return call(*args)
    for i, bad in ((0, 0), (0, 65536), (1, -1), (1, 2**28 + 1), (7, 0), (7, 2**28 + 1), (13, 0), (13, 65), (14, 96), (15, 0), (15, 3),
                   (12, cache(kv4, page_size=48))):
        assert but((i, bad)) == SHAPE, (i, bad)
    for i in (2, 3, 4, 5, 6, 8, 9, 10, 11, 16, 17):
        assert but((i, None)) == NULL, i
    for i in (8, 9, 10, 11):
        assert but((i, SOME + 64), (17, SOME + 64)) == SHAPE, i       # an array that is written and the status as well
    assert but((12, cache(kv4, None))) == NULL and but((12, cache(kv4, ODD))) == ALIGN


def test_a_status_of_another_kind(kv4):  # noqa: F811
    """On the CPU: the first argument that does not live on the GPU is refused, the status like the others."""
    import torch
    ints = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(kv4.ShotKVError, match="status must"):
        kv4.tree_keep(ints[:2], ints, ints, ints, ints[:1], kv4.TreeKept.empty(1, 3, device="cpu"), status=ints[:1])
