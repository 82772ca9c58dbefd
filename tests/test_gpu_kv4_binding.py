"""The binding of the paged 4-bit cache: tensors that change between calls, arguments that are left out."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc
from test_gpu_kv4 import Problem, check_rotated, check_plan, i32, kv4, make_rope, run_plan  # noqa: F401  (kv4 is the fixture)

pytestmark = pytest.mark.gpu


def test_weights_and_tables_of_a_rotation_may_be_given_other_memory(kv4):  # noqa: F811
    T, H, Hkv, D = 5, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn((T, n, D), generator=g, device="cuda") for n in (H, Hkv))
    pos = np.arange(T) * 3
    rope, other = make_rope(kv4, D, D, torch.float32, False, True, 0), make_rope(kv4, D, D, torch.float32, False, True, 1)
    held = [rope.table.data, rope.q_weight.data, rope.k_weight.data]        # what the tensors had stays allocated
    kv4.qk_norm_rope(rope, q, k, i32(pos))
    rope.q_weight.data = other.q_weight.clone()                             # the same tensor, other memory
    rope.table.set_(other.table.clone())
    rope.k_weight = torch.nn.Parameter(other.k_weight.clone(), requires_grad=False)
    q_out, k_out = kv4.qk_norm_rope(rope, q, k, i32(pos))
    check_rotated(q_out, q, other.q_weight, other, pos, torch.float32)
    check_rotated(k_out, k, other.k_weight, other, pos, torch.float32)
    rope.q_weight, rope.eps, rope.interleaved = None, 0.5, True
    q_out, k_out = kv4.qk_norm_rope(rope, q, k, i32(pos))
    check_rotated(q_out, q, None, rope, pos, torch.float32)
    check_rotated(k_out, k, other.k_weight, rope, pos, torch.float32)
    rope.k_weight = other.k_weight.bfloat16()
    with pytest.raises(kv4.ShotKVError, match="k_weight"):
        kv4.qk_norm_rope(rope, q, k, i32(pos))
    del held


def test_pages_may_be_given_other_memory(kv4):  # noqa: F811
    p = Problem(kv4, [70, 33], [1, 1], 4, 2, 64, 32, torch.float32)
    want, held, pages = p.run().clone(), p.cache.pages.data, p.cache.pages.clone()
    p.cache.pages.zero_()
    p.cache.pages.data = pages
    assert torch.equal(p.run(), want) and not held.any()
    p.cache.pages = torch.cat([pages, pages])           # another tensor, of more pages
    assert p.cache.n_pages == 2 * len(pages) and torch.equal(p.run(), want)
    p.table += torch.where(p.table < len(pages), len(pages), 0).int()
    assert torch.equal(p.run(), want)
    p.cache.pages = pages.flatten()[:-1]
    with pytest.raises(kv4.ShotKVError, match="whole number of pages"):
        p.run()
    p.cache.pages = pages.cpu()
    with pytest.raises(kv4.ShotKVError, match="GPU"):
        p.run()


def test_arrays_of_a_plan_may_be_given_other_memory(kv4):  # noqa: F811
    """Between two plans every array moves; what it had stays allocated, and is not written."""
    cached, new, stack, table = [10, 0, 64], [30, 70, 1], np.arange(9), np.array([[20, -1, -1], [-1, -1, -1], [21, 22, -1]])
    names = ("block_table", "free_left", "seq_lens", "query_start", "slot_map", "token_pos", "status")
    plan = run_plan(kv4, 32, cached, new, stack, 9, table, 110)
    ref = orc.pages_plan(32, cached, new, stack, 9, table, 110)
    check_plan(plan, ref)
    held = {}
    for how in ("data", "set"):
        for name in names:
            t = getattr(plan, name)
            held[name] = t.data
            fresh = i32(table) if name == "block_table" else torch.full(t.shape, -77, dtype=torch.int32, device="cuda")
            if how == "data":
                t.data = fresh
            else:
                t.set_(fresh)
        before = {name: t.clone() for name, t in held.items()}
        kv4.pages_plan(32, i32(cached), i32(new), i32(stack), i32([9]), plan)
        check_plan(plan, ref)
        assert all(torch.equal(held[name], before[name]) for name in names)
    plan.slot_map.resize_(50)
    with pytest.raises(kv4.ShotKVError, match="token_pos"):         # of 110 tokens still
        kv4.pages_plan(32, i32(cached), i32(new), i32(stack), i32([9]), plan)


@pytest.mark.parametrize("news", [[2, 3, 1], [9, 40, 5]])
def test_attention_without_max_q_len_takes_all_tokens(kv4, news):  # noqa: F811
    """And rows that no request has are zeros in an output that is made by the call."""
    p = Problem(kv4, [70, 300, 40], news, 8, 2, 128, 64, torch.bfloat16)
    want = p.run()
    args = (p.table, i32(p.lens), p.scale)
    p.check(kv4.attention(p.cache, p.q, *args, i32(p.start)))       # (another bound may be another kernel, whose last bits differ)
    assert torch.equal(kv4.attention(p.cache, p.q, *args, query_start=i32(p.start), max_q_len=max(news)), want)
    torch.full((1 << 20,), 9.0, device="cuda")          # (memory that is handed out next)
    wide = torch.cat([p.q[:4] * 0 + 1, p.q, p.q[:3]])
    for most in (None, max(news)):
        out = kv4.attention(p.cache, wide, *args, i32(p.start + 4), most)
        p.check(out[4:-3])
        assert not out[:4].any() and not out[-3:].any()
    guard = torch.full_like(wide, 5.0)
    assert kv4.attention(p.cache, wide, *args, i32(p.start + 4), None, guard) is guard
    p.check(guard[4:-3])
    assert torch.all(guard[:4] == 5) and torch.all(guard[-3:] == 5)


def test_strides_of_dimensions_of_one_do_not_matter(kv4):  # noqa: F811
    """One token, one head or one problem whose stride is no multiple of anything: the rows are where they would be without it."""
    p = Problem(kv4, [70], [1], 4, 1, 64, 32, torch.bfloat16)
    want, flat = p.run(), p.q.flatten()
    for shape, stride in (((1, 4, 64), (259, 64, 1)), ((1, 1, 4, 64), (7, 259, 64, 1)), ((1, 1, 4, 64), (1, 1, 64, 1))):
        out = torch.zeros(4 * 64, dtype=torch.bfloat16, device="cuda")
        kv4.attention(p.cache, flat.as_strided(shape, stride), p.table, i32(p.lens), p.scale, out=out.as_strided(shape, stride))
        assert torch.equal(out.view(1, 4, 64), want), shape
    k, v = torch.randn((2, 6, 1, 64), device="cuda").bfloat16()
    slots = i32(np.arange(6))
    pools = [torch.zeros((1, kv4.page_bytes(32, 1, 64)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    kv4.store(kv4.Cache(pools[0], 32, 1, 64), k, v, slots)
    for shape, stride in (((6, 1, 64), (64, 3, 1)), ((1, 6, 1, 64), (5, 64, 3, 1)), ((6, 1, 1, 64), (64, 5, 3, 1))):
        pools[1].zero_()
        kv4.store(kv4.Cache(pools[1], 32, 1, 64), k.as_strided(shape, stride), v.as_strided(shape, stride, v.storage_offset()), slots)
        assert torch.equal(pools[0], pools[1]), shape
