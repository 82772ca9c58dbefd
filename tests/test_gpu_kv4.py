"""The paged 4-bit cache on the GPU against its plain 64-bit definitions, through the public binding.

Tolerances.  Codes, scales, tables and maps: equal.  Rotated rows: a few roundings of 32 bits on values of the size of the
row (4e-6 of its largest magnitude) and one rounding to the storage type (2^-8 of the value at most in bf16).  Attention: a
weight is off by 2^-16 as two bf16 numbers, a logit by some 32-bit roundings of terms whose sizes add up to less than 64
(1e-5), so an output is off by that share of the weighted sum of |v|: 5e-5, and by its own rounding.  lse: 2e-5 + 1e-6 of
its size.
"""
import math

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def kv4():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2502_01941_amd import kv4
    kv4.load_library()
    return kv4


def host(t):
    t = t.detach().cpu()
    return (t.float() if t.dtype == torch.bfloat16 else t).numpy()


def i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32, device="cuda").contiguous()


# ---- the cache -------------------------------------------------------------------------------------------

def awkward_rows(rng, shape, dtype):
    """Values of many sizes: zeros of both signs, exact middles, denormals, the largest, and some that are not finite."""
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-12, 12, shape[:-1] + (1,)))
    flat = x.reshape(-1, shape[-1])
    flat[1::7] = rng.integers(-28, 29, flat[1::7].shape) / 4.0
    flat[2::7, :32] = 0.0
    flat[2::7, 1] = -0.0
    flat[3::7] = rng.standard_normal(flat[3::7].shape) * 1e-39
    flat[4::14] = rng.standard_normal(flat[4::14].shape) * 8e37
    flat[5::14, 3] = np.inf
    flat[6::14, 40] = np.nan
    flat[0, 0] = 3.38e38
    return torch.from_numpy(np.clip(x, -3.38e38, 3.38e38)).to(dtype) if not np.isnan(x).any() else \
        torch.from_numpy(np.where(np.isfinite(x), np.clip(x, -3.38e38, 3.38e38), x)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,heads,page,tokens", [(128, 8, 64, 1), (128, 2, 32, 75), (64, 3, 128, 131), (64, 1, 32, 6), (128, 5, 256, 33)])
def test_store_writes_the_defined_bytes_and_load_reads_them(kv4, D, heads, page, tokens, dtype):
    rng = np.random.default_rng(tokens + D)
    n_pages = 3 * tokens // page + 3
    pool = torch.from_numpy(rng.integers(0, 256, (n_pages, orc.page_bytes(page, heads, D)), dtype=np.uint8)).cuda()
    cache = kv4.Cache(pool.clone(), page, heads, D)
    assert cache.n_pages == n_pages and kv4.page_bytes(page, heads, D) == orc.page_bytes(page, heads, D)
    slots = rng.permutation(n_pages * page)[:tokens]
    if tokens > 4:
        slots[2], slots[4] = -1, n_pages * page        # none, and one past the pool: neither is stored
    k, v = (awkward_rows(rng, (tokens, heads, D), TYPES[dtype]).cuda() for _ in range(2))
    kv4.store(cache, k, v, i32(slots))
    want = pool.cpu().numpy().reshape(-1).copy()
    live = (slots >= 0) & (slots < n_pages * page)
    for t in np.nonzero(live)[0]:
        orc.store(want, page, heads, D, int(slots[t]), host(k)[t], host(v)[t])
    np.testing.assert_array_equal(cache.pages.cpu().numpy().reshape(-1), want)
    got_k, got_v = kv4.load(cache, i32(slots), dtype=TYPES[dtype])
    for h in range(heads):
        ref_k, ref_v = orc.load(want, page, heads, D, np.where(live, slots, 0), h)
        np.testing.assert_array_equal(host(got_k)[:, h], np.where(live[:, None], ref_k, 0).astype(np.float32))
        np.testing.assert_array_equal(host(got_v)[:, h], np.where(live[:, None], ref_v, 0).astype(np.float32))


def test_store_takes_rows_of_any_layout(kv4):
    """A cache laid out by head, a slice of a fused projection and dense rows give the same bytes."""
    P, N, H, D = 3, 21, 4, 128
    g = torch.Generator(device="cuda").manual_seed(0)
    k, v = torch.randn((2, P, H, N, D), generator=g, device="cuda").bfloat16()
    slots = i32(np.random.default_rng(0).permutation(128)[:P * N])
    pools = [torch.zeros((2, kv4.page_bytes(64, H, D)), dtype=torch.uint8, device="cuda") for _ in range(3)]
    kt, vt = k.transpose(1, 2), v.transpose(1, 2)
    kv4.store(kv4.Cache(pools[0], 64, H, D), kt, vt, slots)
    kv4.store(kv4.Cache(pools[1], 64, H, D), kt.reshape(P * N, H, D), vt.reshape(P * N, H, D), slots)
    fused = torch.cat([kt.reshape(P * N, H, D), vt.reshape(P * N, H, D)], dim=1)
    kv4.store(kv4.Cache(pools[2], 64, H, D), fused[:, :H], fused[:, H:], slots)
    assert torch.equal(pools[0], pools[1]) and torch.equal(pools[0], pools[2]) and pools[0].any()
    out = torch.zeros((P, H, N, D), dtype=torch.bfloat16, device="cuda")
    out_v = torch.zeros_like(out)
    kv4.load(kv4.Cache(pools[0], 64, H, D), slots, out.transpose(1, 2), out_v.transpose(1, 2))
    dense_k, dense_v = kv4.load(kv4.Cache(pools[0], 64, H, D), slots)
    assert torch.equal(out.transpose(1, 2).reshape(P * N, H, D), dense_k)
    assert torch.equal(out_v.transpose(1, 2).reshape(P * N, H, D), dense_v)


# ---- page tables -----------------------------------------------------------------------------------------

def run_plan(kv4, page, cached, new, stack, count, table, tokens, pos=None, share=0):
    plan = kv4.PagePlan.empty(i32(table), tokens)
    for t in (plan.free_left, plan.seq_lens, plan.query_start, plan.slot_map, plan.token_pos, plan.status):
        t.fill_(-77)
    kv4.pages_plan(page, i32(cached), i32(new), i32(stack), i32([count]), plan, None if pos is None else i32(pos), share)
    return plan


def check_plan(plan, ref):
    for name in ("block_table", "seq_lens", "query_start", "slot_map", "token_pos", "status"):
        np.testing.assert_array_equal(getattr(plan, name).cpu().numpy(), ref[name], err_msg=name)
    assert int(plan.free_left) == ref["free_left"]


@pytest.mark.parametrize("R,page,most,share,tight", [(1, 32, 1, 0, 0), (16, 64, 1, 0, 0), (7, 32, 300, 0, 0), (300, 32, 90, 0, 0),
                                                     (300, 64, 90, 0, 40), (5, 128, 500, 512, 0), (600, 32, 3, 4, 30), (64, 64, 0, 0, 0)])
def test_plan(kv4, R, page, most, share, tight):
    rng = np.random.default_rng(R + page)
    cached, new = rng.integers(0, 400, R), rng.integers(0, most + 1, R)
    cached[::3] = cached[::3] // page * page        # full pages too
    held, need = -(-cached // page), -(-(cached + new) // page)
    max_pages = int(need.max()) + 1
    pool = rng.permutation(int(need.sum()) + 3)
    table = np.full((R, max_pages), -1)
    at = 0
    for r in range(R):
        table[r, :held[r]] = pool[at:at + held[r]]
        at += held[r]
    count = max(0, len(pool) - at - tight)
    stack = np.concatenate([pool[at:], np.zeros(1, int)])
    tokens = R * share + 5 if share else int(new.sum()) + 5
    pos = rng.integers(0, 10000, R) if share else None
    ref = orc.pages_plan(page, cached, new, stack, count, table, tokens, pos, share)
    if tight:
        assert set(ref["status"]) == {0, -4}
    check_plan(run_plan(kv4, page, cached, new, stack, count, table, tokens, pos, share), ref)


def test_plan_refuses_lengths_that_make_no_sense(kv4):
    cached = [10, -3, 60, 5, 2**31 - 1, 40, 0, 3]
    new = [5, 4, 10, -2, 2**31 - 1, 9, 30, 0]
    table = np.arange(16).reshape(8, 2)
    stack = np.arange(100, 120)
    for tokens in (100, 40, 3):
        ref = orc.pages_plan(32, cached, new, stack, 20, table, tokens)
        got = run_plan(kv4, 32, cached, new, stack, 20, table, tokens)
        ref["query_start"] = np.minimum(ref["query_start"], 2**31 - 1)
        check_plan(got, ref)
    share = 8
    ref = orc.pages_plan(32, cached, new, stack, 20, table, 64, None, share)
    ref["query_start"] = np.minimum(ref["query_start"], 2**31 - 1)
    check_plan(run_plan(kv4, 32, cached, new, stack, 20, table, 64, None, share), ref)


def test_a_count_past_the_stack_counts_its_pages(kv4):
    """More pages than the stack has room for are not there."""
    stack = np.random.default_rng(3).permutation(7)
    for count in (8, 10**6, 2**31 - 1, 7, -3):
        table = np.full((4, 4), -1)
        plan = run_plan(kv4, 32, [0, 31, 64, 0], [70, 2, 32, 64], stack, count, table, 168)
        ref = orc.pages_plan(32, [0, 31, 64, 0], [70, 2, 32, 64], stack, min(max(count, 0), 7), table, 168)
        check_plan(plan, ref)


def test_release_is_the_inverse_and_leaves_others(kv4):
    rng = np.random.default_rng(9)
    R, page = 290, 32
    new = rng.integers(0, 200, R)
    stack = rng.permutation(3000)
    plan = run_plan(kv4, page, np.zeros(R, int), new, stack, 2500, np.full((R, 8), -1), int(new.sum()))
    ref = orc.pages_plan(page, np.zeros(R, int), new, stack, 2500, np.full((R, 8), -1), int(new.sum()))
    check_plan(plan, ref)
    for finished in (rng.random(R) < 0.4, np.ones(R, bool)):
        lens, table, free, count = plan.seq_lens.clone(), plan.block_table.clone(), i32(stack), plan.free_left.clone()
        kv4.pages_release(page, torch.from_numpy(finished.astype(np.uint8)).cuda(), lens, table, free, count)
        want = orc.pages_release(page, finished, ref["seq_lens"], ref["block_table"], stack, ref["free_left"])
        for got, w in zip((lens, table, free), want):
            np.testing.assert_array_equal(got.cpu().numpy(), w)
        assert int(count) == want[3]
    np.testing.assert_array_equal(free.cpu().numpy(), stack)


# ---- norms and rotation ----------------------------------------------------------------------------------

def make_rope(kv4, D, rot, dtype, interleaved, norm, seed=0, positions=700):
    g = torch.Generator().manual_seed(seed)
    angle = torch.rand((positions, rot // 2), generator=g, dtype=torch.float64) * 6.2831
    table = torch.cat([angle.cos(), angle.sin()], dim=1).float().cuda()
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(dtype).cuda() if norm else None for _ in range(2)]
    return kv4.Rope(table, w[0], w[1], 1e-5, interleaved)


def check_rotated(got, x, weight, rope, pos, dtype):
    x, got, table = host(x).astype(np.float64), host(got), host(rope.table).astype(np.float64)
    half = table.shape[1] // 2
    for t in range(len(x)):
        for h in range(x.shape[1]):
            if not 0 <= pos[t] < len(table):
                assert not got[t, h].any()
                continue
            ref = orc.norm_rope(x[t, h], None if weight is None else host(weight), rope.c.eps, table[pos[t], :half],
                                table[pos[t], half:], bool(rope.c.interleaved))
            tol = 4e-6 * np.abs(ref).max() + (np.abs(ref) * 2.0 ** -8 if dtype == torch.bfloat16 else 0)
            assert np.all(np.abs(got[t, h] - ref) <= tol), (t, h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H,Hkv,D,rot,interleaved,norm", [
    (1, 4, 4, 128, 128, False, True), (5, 32, 8, 128, 128, False, True), (9, 8, 1, 128, 64, False, True),
    (17, 7, 1, 128, 128, True, True), (3, 6, 2, 64, 64, False, False), (33, 5, 5, 64, 32, True, True), (4, 3, 3, 128, 96, False, True),
    (2, 8, 2, 64, 16, False, True)])
def test_norm_rope(kv4, T, H, Hkv, D, rot, interleaved, norm, dtype):
    dt = TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(T)
    qkv = (torch.randn((T, H + 2 * Hkv, D), generator=g, device="cuda") * 3).to(dt)
    rope = make_rope(kv4, D, rot, dt, interleaved, norm, T)
    pos = np.random.default_rng(T).integers(0, 700, T)
    if T > 3:
        pos[1], pos[3] = -1, 700        # padding
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    q_out, k_out = kv4.qk_norm_rope(rope, q, k, i32(pos))
    check_rotated(q_out, q, rope.q_weight, rope, pos, dt)
    check_rotated(k_out, k, rope.k_weight, rope, pos, dt)
    # by head, and only the values kept: the same numbers
    by_head = torch.full((H, T, D), 9.0, dtype=dt, device="cuda"), torch.full((Hkv, T, D), 9.0, dtype=dt, device="cuda")
    kv4.qk_norm_rope(rope, q, k, i32(pos), by_head[0].transpose(0, 1), by_head[1].transpose(0, 1))
    assert torch.equal(by_head[0].transpose(0, 1), q_out) and torch.equal(by_head[1].transpose(0, 1), k_out)
    # into the cache in the same call: the bytes that a store of the rows makes, and nothing for padding or without a slot
    slots = np.random.default_rng(T + 1).permutation(8 * 32)[:T] if T <= 256 else None
    if T > 4:
        slots[0] = -1
    pools = [torch.full((8, kv4.page_bytes(32, Hkv, D)), 7, dtype=torch.uint8, device="cuda") for _ in range(2)]
    q2, k2 = kv4.qk_norm_rope(rope, q, k, i32(pos), None, None, v, kv4.Cache(pools[0], 32, Hkv, D), i32(slots))
    assert k2 is None and torch.equal(q2, q_out)
    kept = np.where((pos >= 0) & (pos < 700), slots, -1)
    kv4.store(kv4.Cache(pools[1], 32, Hkv, D), k_out, v, i32(kept))
    assert torch.equal(pools[0], pools[1])
    # both outputs at once
    _, k3 = kv4.qk_norm_rope(rope, q, k, i32(pos), None, torch.empty_like(k_out), v, kv4.Cache(pools[0], 32, Hkv, D), i32(slots))
    assert torch.equal(k3, k_out) and torch.equal(pools[0], pools[1])


def test_norm_rope_of_a_long_prompt(kv4):
    """Many workgroups, rows of every size: each row against the same row on its own."""
    T, H, Hkv, D = 1201, 16, 2, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    x = (torch.randn((T, H + Hkv, D), generator=g, device="cuda") * torch.logspace(-6, 6, T, device="cuda")[:, None, None]).bfloat16()
    rope = make_rope(kv4, D, D, torch.bfloat16, False, True)
    pos = np.arange(T) % 700
    q_out, k_out = kv4.qk_norm_rope(rope, x[:, :H], x[:, H:], i32(pos))
    rows = np.concatenate([np.arange(4), np.random.default_rng(0).integers(0, T, 12), np.arange(T - 4, T)])
    at = torch.from_numpy(rows).cuda()
    check_rotated(q_out[at], x[at, :H], rope.q_weight, rope, pos[rows], torch.bfloat16)
    check_rotated(k_out[at], x[at, H:], rope.k_weight, rope, pos[rows], torch.bfloat16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,rot,interleaved", [(128, 128, False), (64, 64, False), (128, 64, False), (64, 48, False), (128, 32, True)])
def test_norms_of_one_kind_in_place(kv4, D, rot, interleaved, dtype):
    """Weights for queries or for keys alone, head counts that nothing divides, outputs in the place of inputs, and padding whose
    rows are not finite."""
    T, H, Hkv, dt = 2500, 10, 5, TYPES[dtype]
    both = make_rope(kv4, D, rot, dt, interleaved, True, rot)
    g = torch.Generator(device="cuda").manual_seed(rot + D)
    pos = np.random.default_rng(rot).integers(0, 700, T)
    pos[[0, 77, 2499]] = [-1, 700, 2**31 - 1]
    at = np.r_[0:3, 76:79, 1200:1203, 2497:2500]
    for weights in ((both.q_weight, None), (None, both.k_weight)):
        rope = kv4.Rope(both.table, *weights, 1e-5, interleaved)
        x = (torch.randn((T, H + Hkv, D), generator=g, device="cuda") * 3).to(dt)
        x[0], x[77], x[2499] = float("nan"), float("inf"), float("-inf")
        before = x[at].clone()
        q, k = kv4.qk_norm_rope(rope, x[:, :H], x[:, H:], i32(pos), x[:, :H], x[:, H:])
        check_rotated(q[at], before[:, :H], weights[0], rope, pos[at], dt)
        check_rotated(k[at], before[:, H:], weights[1], rope, pos[at], dt)


# ---- attention -------------------------------------------------------------------------------------------

class Problem:
    """Requests over pages in a random order, with garbage wherever no token of theirs is."""

    def __init__(self, kv4, lens, news, H, Hkv, D, page, dtype, seed=0, spread=2.0, garbage=255, extra_pages=2, values=None):
        rng = np.random.default_rng(seed)
        self.kv4, self.lens, self.news, self.G, self.D = kv4, list(lens), list(news), H // Hkv, D
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + extra_pages
        order = rng.permutation(n_pages)
        max_pages = max(max(need), 1) + 1
        table = np.full((len(lens), max_pages), 2**31 - 1)
        at = 0
        for r, n in enumerate(need):
            table[r, :n] = order[at:at + n]
            at += n
        self.cache = kv4.Cache(torch.full((n_pages, kv4.page_bytes(page, Hkv, D)), garbage, dtype=torch.uint8, device="cuda"),
                               page, Hkv, D)
        slots = np.concatenate([table[r, np.arange(n) // page] * page + np.arange(n) % page for r, n in enumerate(lens)]).astype(np.int64)
        self.slots = slots
        k, v = rng.standard_normal((2, len(slots), Hkv, D))
        if values is not None:
            values(k, v)
        if len(slots):
            kv4.store(self.cache, torch.from_numpy(k).float().cuda(), torch.from_numpy(v).float().cuda(), i32(slots))
            kk, vv = kv4.load(self.cache, i32(slots), dtype=torch.float32)
            self.k, self.v = host(kk).astype(np.float64), host(vv).astype(np.float64)
        else:
            self.k = self.v = np.zeros((0, Hkv, D))
        self.table, self.start = i32(table), np.concatenate([[0], np.cumsum(news)])
        self.q = torch.from_numpy(rng.standard_normal((int(self.start[-1]), H, D)) * spread).to(dtype).cuda()
        self.dtype, self.scale, self.H, self.Hkv = dtype, 1 / math.sqrt(D), H, Hkv

    def run(self, **kw):
        T = len(self.q)
        self.lse = torch.full((T, self.H), 99.0, device="cuda")
        return self.kv4.attention(self.cache, self.q, self.table, i32(self.lens), self.scale, i32(self.start), max(max(self.news), 1),
                                  None, self.lse, **kw)

    def check(self, out, lse=None, requests=None):
        lse = host(self.lse if lse is None else lse)
        out, q = host(out), host(self.q).astype(np.float64)
        share = 5e-5
        first = np.concatenate([[0], np.cumsum(self.lens)])
        for r in range(len(self.lens)) if requests is None else requests:
            mine = slice(self.start[r], self.start[r + 1])
            for g in range(self.Hkv):
                heads = slice(g * self.G, (g + 1) * self.G)
                k, v = self.k[first[r]:first[r + 1], g], self.v[first[r]:first[r + 1], g]
                ref, ref_lse, spread = orc.attention(q[mine, heads], k, v, self.news[r], self.scale)
                tol = share * spread + (np.abs(ref) * 2.0 ** -8 if self.dtype == torch.bfloat16 else 0)
                assert np.all(np.abs(out[mine, heads] - ref) <= tol + 1e-30), (r, g, np.abs(out[mine, heads] - ref).max())
                got = lse[mine, heads]
                np.testing.assert_array_equal(np.isneginf(got), np.isneginf(ref_lse))
                seen = np.isfinite(ref_lse)
                assert np.all(np.abs(got[seen] - ref_lse[seen]) <= 2e-5 + 1e-6 * np.abs(ref_lse[seen])), (r, g)


EDGES = [0, 1, 2, 31, 32, 33, 63, 64, 65, 95, 127, 128, 129, 257, 500]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D,page", [(32, 8, 128, 64), (8, 1, 128, 32), (7, 1, 64, 128), (5, 5, 64, 32), (12, 2, 128, 256)])
def test_single_tokens(kv4, H, Hkv, D, page, dtype):
    p = Problem(kv4, EDGES, [1] * len(EDGES), H, Hkv, D, page, TYPES[dtype], seed=D + H)
    p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D,most", [(32, 8, 128, 2), (8, 2, 128, 4), (4, 1, 64, 8), (14, 2, 128, 3), (3, 3, 64, 16), (8, 1, 128, 5)])
def test_drafts(kv4, H, Hkv, D, most, dtype):
    """A few tokens per request, fewer in the cache than new ones among them (rows that see nothing), and none."""
    rng = np.random.default_rng(most)
    news = [most, 0, 1, most, most] + rng.integers(0, most + 1, 10).tolist()
    p = Problem(kv4, EDGES, news, H, Hkv, D, 32, TYPES[dtype], seed=most)
    out = p.run()
    p.check(out)
    assert np.isneginf(host(p.lse)[:most]).all() and not host(out)[:most].any()     # a request without a token in the cache


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D,lens,news", [
    (8, 2, 128, [300, 77, 40], [300, 20, 40]), (4, 1, 64, [515, 130], [100, 130]), (7, 1, 128, [200, 33], [65, 33]),
    (8, 8, 128, [129], [129]), (8, 1, 64, [64, 1, 100], [64, 1, 1])])
def test_chunks_of_prompts(kv4, H, Hkv, D, lens, news, dtype):
    p = Problem(kv4, lens, news, H, Hkv, D, 64, TYPES[dtype], seed=sum(lens))
    p.check(p.run())


@pytest.mark.parametrize("lens,news", [([3277], [1]), ([9000, 5, 4096, 1], [1, 1, 1, 1]), ([5000, 700], [3, 2]), ([2500], [70])])
def test_long_caches_are_shared_by_workgroups(kv4, lens, news):
    p = Problem(kv4, lens, news, 8, 2, 128, 64, torch.bfloat16, seed=len(lens))
    p.check(p.run())
    q = Problem(kv4, lens, news, 4, 1, 64, 32, torch.float32, seed=len(lens))
    q.check(q.run())


def test_many_requests(kv4):
    lens = np.random.default_rng(0).integers(0, 90, 700)
    p = Problem(kv4, lens, [1] * 700, 4, 2, 64, 32, torch.bfloat16)
    p.check(p.run())


def test_peaked_and_flat_rows(kv4):
    """Logits of several hundred and equal ones; a key far ahead of the others late in the cache, and early."""
    for spread in (0.0, 1e-3, 60.0):
        p = Problem(kv4, [700, 33], [1, 1], 8, 2, 128, 64, torch.float32, spread=spread)
        out = p.run()
        if spread < 1:
            p.check(out)
            continue
        # logits of 700: their 32-bit roundings are the error (2^-23 * 700 per sum of terms)
        p_out, ref = host(out), []
        first = 0
        for r, n in enumerate(p.lens):
            for g in range(2):
                o, _, s = orc.attention(host(p.q).astype(np.float64)[r:r + 1, 4 * g:4 * g + 4], p.k[first:first + n, g], p.v[first:first + n, g], 1, p.scale)
                assert np.all(np.abs(p_out[r, 4 * g:4 * g + 4] - o[0]) <= 2e-3 * np.abs(p.v).max())
            first += n


def test_values_of_all_sizes(kv4):
    def values(k, v):
        v *= np.exp(np.random.default_rng(1).uniform(-60, 60, (1, v.shape[1], v.shape[2])))
        k[:, :, ::3] *= 30
    p = Problem(kv4, [400, 65, 7], [1, 1, 1], 8, 2, 128, 64, torch.float32, values=values, spread=0.3)
    p.check(p.run())


def test_what_a_row_does_not_see_does_not_reach_it(kv4):
    """A token whose keys and values are not finite: rows before it are what they are without it, those from it on are NaN."""
    for D, dtype in ((128, torch.bfloat16), (64, torch.float32)):
        def values(k, v):
            k[100], v[100, :, 40:] = np.nan, np.inf
        p = Problem(kv4, [105], [10], 4, 2, D, 32, dtype, values=values)
        out, lse = host(p.run()), host(p.lse)
        assert np.isfinite(out[:5]).all() and np.isnan(out[5:]).all() and np.isnan(lse[5:]).all()
        p.lens, p.news, p.start, p.k, p.v, q = [100], [5], np.array([0, 5]), p.k[:100], p.v[:100], p.q
        p.q = q[:5]
        p.check(torch.from_numpy(out[:5]), torch.from_numpy(lse[:5]))

        def only_values(k, v):
            v[100, :, 40:] = np.inf         # its group of channels and those behind, of the rows that see it
        p = Problem(kv4, [105], [10], 4, 2, D, 32, dtype, values=only_values)
        out = host(p.run())
        assert np.isfinite(out[:5]).all() and np.isfinite(out[5:, :, :32]).all() and np.isnan(out[5:, :, 32:]).all()
        assert np.isfinite(host(p.lse)).all()


def test_queries_that_are_not_finite_stay_in_their_rows(kv4):
    p = Problem(kv4, [90, 40], [4, 1], 8, 2, 128, 64, torch.bfloat16)
    p.q[1, 3] = float("nan")
    p.q[4, 0, 5] = float("inf")
    out = host(p.run())
    assert np.isnan(out[1, 3]).all() and np.isnan(out[4, 0]).all()
    out[1, 3] = out[4, 0] = 0
    assert np.isfinite(out).all()


def test_lists_that_name_no_page(kv4):
    """Entries outside the pool are tokens that nobody sees; lengths past the table are cut."""
    p = Problem(kv4, [160, 160], [1, 1], 4, 2, 128, 32, torch.float32)
    p.table[0, 1], p.table[0, 4] = -5, 10**6
    out = p.run()
    keep = np.r_[0:32, 64:128]
    k, v = p.k.copy(), p.v.copy()
    for g in range(2):
        ref, lse, s = orc.attention(host(p.q).astype(np.float64)[:1, 2 * g:2 * g + 2], k[keep, g], v[keep, g], 1, p.scale)
        assert np.all(np.abs(host(out)[:1, 2 * g:2 * g + 2] - ref) <= 5e-5 * s)
        assert np.all(np.abs(host(p.lse)[:1, 2 * g:2 * g + 2] - lse) <= 2e-5)
    p.check(out, requests=[1])
    whole = p.run()
    table = p.table[:, :5].contiguous()
    cut = kv4.attention(p.cache, p.q, table, i32([160, 10**9]), p.scale, None)
    assert torch.equal(cut, whole)


def test_pages_that_requests_share(kv4):
    p = Problem(kv4, [96, 96, 96], [1, 1, 1], 4, 2, 64, 32, torch.float32)
    p.table[1, :2] = p.table[0, :2]         # a common prefix of two pages
    for a in (p.k, p.v):
        a[96:96 + 64] = a[:64]
    p.check(p.run())


def test_rows_of_any_layout_and_no_lse(kv4):
    p = Problem(kv4, [70, 300], [2, 2], 8, 2, 128, 64, torch.bfloat16)
    want = p.run()
    wide = torch.zeros((4, 12, 128), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:10] = p.q
    out = torch.zeros((8, 4, 128), dtype=torch.bfloat16, device="cuda")
    kv4.attention(p.cache, wide[:, 2:10], p.table, i32(p.lens), p.scale, i32(p.start), 2, out.transpose(0, 1))
    assert torch.equal(out.transpose(0, 1), want)
    four = p.q.view(2, 2, 8, 128)
    got = kv4.attention(p.cache, four, p.table, i32(p.lens), p.scale, i32(p.start), 2)
    assert got.shape == four.shape and torch.equal(got.view(4, 8, 128), want)


def test_starts_that_run_past_the_batch_write_nothing_there(kv4):
    p = Problem(kv4, [70, 300, 40], [2, 3, 1], 8, 2, 128, 64, torch.bfloat16)
    want, guard = p.run(), torch.full((9, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    kv4.attention(p.cache, p.q, p.table, i32(p.lens), p.scale, i32([0, 2, 5, 2**31 - 1]), 3, guard[:6])
    assert torch.equal(guard[:6], want) and torch.all(guard[6:] == 5)
    guard.fill_(5.0)
    kv4.attention(p.cache, p.q, p.table, i32(p.lens), p.scale, i32([0, 2, 5, 6]), 2, guard[:6])    # max_q_len cuts the second
    assert torch.equal(guard[0:2], want[0:2]) and torch.all(guard[4] == 5) and torch.equal(guard[5], want[5])


def test_a_pool_of_more_than_4_gib(kv4):
    """Offsets past 32 bits: a request whose pages lie at the end of a pool of 5 GiB."""
    D, H, page = 128, 8, 128
    n_pages = 5 * 2**30 // kv4.page_bytes(page, H, D)
    cache = kv4.Cache.empty(n_pages, page, H, D)
    table = i32([[n_pages - 1, 0, n_pages - 3]])
    slots = np.concatenate([(n_pages - 1) * page + np.arange(128), np.arange(128), (n_pages - 3) * page + np.arange(44)])
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = torch.randn((2, 300, H, D), generator=g, device="cuda")
    kv4.store(cache, k, v, i32(slots))
    kk, vv = kv4.load(cache, i32(slots), dtype=torch.float32)
    q = torch.randn((1, H, D), generator=g, device="cuda")
    out = host(kv4.attention(cache, q, table, i32([300]), 0.1))
    for h in range(H):
        ref, _, s = orc.attention(host(q)[:, h:h + 1], host(kk)[:, h].astype(np.float64), host(vv)[:, h].astype(np.float64), 1, 0.1)
        assert np.all(np.abs(out[:, h:h + 1] - ref) <= 5e-5 * s)


def test_results_repeat_bit_for_bit_whatever_the_workspace_held(kv4):
    p = Problem(kv4, [4000, 3, 900, 64], [1, 1, 1, 1], 32, 8, 128, 64, torch.bfloat16)
    ws = kv4.attention_workspace(p.cache, p.q, p.table, 1)
    first = p.run(workspace=ws).clone()
    lse = p.lse.clone()
    ws.fill_(255)
    assert torch.equal(p.run(workspace=ws), first) and torch.equal(p.lse, lse)


# ---- streams, graphs, refusals ---------------------------------------------------------------------------

def decode_step(kv4, s):
    """One decoding step of a layer on static buffers: pages, norms and rotation into the cache, attention."""
    kv4.pages_plan(32, s["lens"], s["one"], s["free"], s["count"], s["plan"], s["pos"])
    qkv, H, Hkv = s["qkv"], s["H"], s["Hkv"]
    kv4.qk_norm_rope(s["rope"], qkv[:, :H], qkv[:, H:H + Hkv], s["plan"].token_pos, s["q"], None, qkv[:, H + Hkv:], s["cache"],
                     s["plan"].slot_map)
    kv4.attention(s["cache"], s["q"], s["plan"].block_table, s["plan"].seq_lens, 0.1, None, 1, s["out"], s["lse"], s["ws"])
    s["lens"].copy_(s["plan"].seq_lens)
    s["count"].copy_(s["plan"].free_left)
    s["pos"].add_(1)


def make_step(kv4):
    R, H, Hkv, D = 6, 8, 2, 128
    cache = kv4.Cache(torch.zeros((40, kv4.page_bytes(32, Hkv, D)), dtype=torch.uint8, device="cuda"), 32, Hkv, D)
    s = {"lens": i32([0] * R), "one": i32([1] * R), "free": i32(np.arange(40)[::-1].copy()), "count": i32([40]), "H": H, "Hkv": Hkv,
         "plan": kv4.PagePlan.empty(i32(np.full((R, 5), -1)), R), "pos": i32(np.arange(R) * 50), "cache": cache,
         "rope": make_rope(kv4, D, D, torch.bfloat16, False, True), "qkv": torch.zeros((R, H + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda"),
         "q": torch.zeros((R, H, D), dtype=torch.bfloat16, device="cuda"), "out": torch.zeros((R, H, D), dtype=torch.bfloat16, device="cuda"),
         "lse": torch.zeros((R, H), device="cuda")}
    s["ws"] = kv4.attention_workspace(cache, s["q"], s["plan"].block_table, 1)
    return s


def test_a_decoding_step_in_a_graph(kv4):
    """Captured once, replayed over steps that cross pages, with eager work between; each replay against an eager twin."""
    eager, graphed = make_step(kv4), make_step(kv4)
    g = torch.Generator(device="cuda").manual_seed(0)
    inputs = [torch.randn(eager["qkv"].shape, generator=g, device="cuda").bfloat16() for _ in range(40)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s in (eager, graphed):          # a first step of both outside of the capture
            s["qkv"].copy_(inputs[0])
            decode_step(kv4, s)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode_step(kv4, graphed)
    for i in range(1, 40):
        eager["qkv"].copy_(inputs[i])
        graphed["qkv"].copy_(inputs[i])
        decode_step(kv4, eager)
        graph.replay()
        if i % 5 == 0:
            torch.cuda.synchronize()
        for name in ("out", "lse", "lens", "count"):
            assert torch.equal(eager[name], graphed[name]), (i, name)
        assert torch.equal(eager["plan"].block_table, graphed["plan"].block_table)
        assert torch.equal(eager["cache"].pages, graphed["cache"].pages)
    assert eager["lens"].tolist() == [40] * 6 and int(eager["count"]) == 40 - 12


def test_calls_follow_their_stream(kv4):
    """Inputs that a stream is still writing when the call is made."""
    p = Problem(kv4, [2000, 1500], [1, 1], 8, 2, 128, 64, torch.bfloat16)
    want, q = p.run().clone(), p.q.clone()
    side = torch.cuda.Stream()
    late = torch.zeros_like(q)
    big = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big * 1e-3
        late.copy_(q)
        out = kv4.attention(p.cache, late, p.table, i32(p.lens), p.scale)
    side.synchronize()
    assert torch.equal(out, want)


def test_refusals(kv4):
    E = kv4.ShotKVError
    p = Problem(kv4, [70], [1], 8, 2, 128, 64, torch.bfloat16)
    lens = i32([70])
    with pytest.raises(E, match="bfloat16|dtype"):
        kv4.attention(p.cache, p.q.half(), p.table, lens, 0.1)
    with pytest.raises(E, match="shape"):
        kv4.attention(p.cache, p.q[:, :, :64], p.table, lens, 0.1)
    with pytest.raises(E, match="unsupported"):
        kv4.attention(p.cache, p.q, p.table, lens, -1.0)
    with pytest.raises(E, match="unsupported"):
        kv4.attention(p.cache, torch.cat([p.q] * 3, dim=1), p.table, lens, 0.1)       # 12 heads per KV head
    with pytest.raises(E, match="int32"):
        kv4.attention(p.cache, p.q, p.table, lens.long(), 0.1)
    with pytest.raises(E, match="workspace"):
        kv4.attention(p.cache, p.q, p.table, lens, 0.1, workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(E, match="aligned"):
        kv4.attention(p.cache, torch.zeros(8 * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(1, 8, 128), p.table, lens, 0.1)
    with pytest.raises(E, match="dense"):
        kv4.attention(p.cache, p.q.repeat(1, 1, 2)[:, :, ::2], p.table, lens, 0.1)
    with pytest.raises(E, match="GPU"):
        kv4.attention(p.cache, p.q.cpu(), p.table, lens, 0.1)
    with pytest.raises(E, match="unsupported"):
        kv4.attention(p.cache, torch.cat([p.q] * 2), p.table, lens, 0.1)              # two tokens, one request, no starts
    with pytest.raises(E):
        kv4.Cache(torch.zeros(100, dtype=torch.uint8, device="cuda"), 64, 2, 128)
    for bad in ((48, 2, 128), (64, 2, 96), (16, 2, 128), (64, 0, 128)):
        with pytest.raises(E):
            kv4.page_bytes(*bad)
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(E, match="shape"):
        kv4.store(p.cache, k, k, i32([0, 1]))
    with pytest.raises(E, match="tokens"):
        kv4.store(p.cache, k, k[:2], i32([0, 1, 2]))
    rope = make_rope(kv4, 128, 128, torch.bfloat16, False, True)
    q3, pos = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda"), i32([0, 1, 2])
    with pytest.raises(E, match="NULL"):
        kv4.qk_norm_rope(rope, q3, k, pos, None, None, k, p.cache, None)              # a cache, and no slots
    with pytest.raises(E, match="weight"):
        kv4.qk_norm_rope(rope, q3.float(), k.float(), pos)
    with pytest.raises(E, match="unsupported"):
        kv4.qk_norm_rope(kv4.Rope(torch.zeros((4, 24), device="cuda")), q3, k, pos)   # 24 channels that turn
    table = i32([[0, 1]])
    plan = kv4.PagePlan.empty(table, 4)
    with pytest.raises(E, match="unsupported"):
        kv4.pages_plan(33, i32([0]), i32([1]), i32([0, 1]), i32([2]), plan)
    plan.free_left = count = i32([2])
    with pytest.raises(E, match="unsupported"):                                       # one word for both counts
        kv4.pages_plan(64, i32([0]), i32([1]), i32([0, 1]), count, plan)
    torch.cuda.synchronize()


def test_batches_of_nothing(kv4):
    """No tokens: every call returns, and nothing is touched."""
    cache = kv4.Cache(torch.full((2, kv4.page_bytes(32, 2, 64)), 9, dtype=torch.uint8, device="cuda"), 32, 2, 64)
    none, none_q = torch.zeros((0, 2, 64), device="cuda"), torch.zeros((0, 4, 64), device="cuda")
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    kv4.store(cache, none, none, empty)
    assert kv4.load(cache, empty, dtype=torch.float32)[0].shape == (0, 2, 64)
    q, k = kv4.qk_norm_rope(make_rope(kv4, 64, 64, torch.float32, False, True), none_q, none, empty)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    out = kv4.attention(cache, none_q, i32([[0], [1]]), i32([5, 0]), 0.1, i32([0, 0, 0]), 1)
    assert out.shape == (0, 4, 64) and torch.all(cache.pages == 9)
    plan = run_plan(kv4, 32, [5, 64], [0, 0], np.arange(3), 3, np.array([[0, -1], [1, 2]]), 0)
    assert plan.seq_lens.tolist() == [5, 64] and int(plan.free_left) == 3 and plan.query_start.tolist() == [0, 0, 0]


def test_mixed_batches(kv4):
    """Chunks of prompts, drafts and single tokens in one call, with requests that have none between."""
    lens, news = [300, 1000, 0, 70, 33, 2000, 90, 512], [150, 1, 0, 5, 33, 1, 0, 200]
    for dtype, D in ((torch.bfloat16, 128), (torch.float32, 64)):
        p = Problem(kv4, lens, news, 8, 2, D, 64, dtype, seed=D)
        p.check(p.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv,D,news", [(8, 2, 128, [9, 16, 12]), (6, 1, 64, [7, 10, 6]), (3, 3, 128, [33, 64, 40]), (8, 1, 64, [5, 8, 7])])
def test_up_to_64_rows(kv4, H, Hkv, D, news, dtype):
    """Rows of two waves, whose tokens four waves share: caches of less than one step, of odd blocks and of many workgroups."""
    for lens in ([33, 64, 40], [95, 97, 64], [2050, 700, 64]):
        p = Problem(kv4, lens, news, H, Hkv, D, 32, TYPES[dtype], seed=len(news) + D)
        p.check(p.run())
    p = Problem(kv4, [3001], news[:1], H, Hkv, D, 64, TYPES[dtype], seed=D)
    p.check(p.run())

    def values(k, v):
        v[70, :, 40:] = np.inf
    p = Problem(kv4, [150], news[1:2], H, Hkv, D, 32, TYPES[dtype], values=values)
    out = host(p.run())
    assert np.isfinite(out[:, :, :32]).all() and np.isnan(out[:, :, 32:]).all()      # channels 40 on: all groups but the first


@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.float32)])
def test_mixed_batches_over_wide_tables(kv4, D, dtype):
    """Tables wide enough that short requests have a kernel of their own next to the chunks."""
    lens, news = [300, 1000, 0, 70, 33, 2000, 90, 512], [150, 1, 0, 8, 33, 1, 0, 9]
    p = Problem(kv4, lens, news, 8, 2, D, 64, dtype, seed=D + 1)
    p.table = torch.cat([p.table, torch.full((len(lens), 1000), 2**31 - 1, dtype=torch.int32, device="cuda")], dim=1)
    p.check(p.run())


def test_chunks_that_many_workgroups_share(kv4):
    """Tiles cut within the cache, groups that fill no tile evenly, values that are not finite in a chunk's own tokens."""
    p = Problem(kv4, [5000], [77], 14, 2, 128, 64, torch.bfloat16, seed=4)
    p.check(p.run())
    p = Problem(kv4, [3000, 200], [50, 200], 10, 2, 64, 32, torch.float32, seed=5)
    p.check(p.run())

    def values(k, v):
        k[100], v[100, :, 40:] = np.nan, np.inf
    for D, dtype in ((128, torch.bfloat16), (64, torch.float32)):
        p = Problem(kv4, [150], [80], 4, 2, D, 32, dtype, values=values)
        out, lse = host(p.run()), host(p.lse)
        assert np.isfinite(out[:30]).all() and np.isnan(out[30:]).all() and np.isnan(lse[30:]).all()
        p.lens, p.news, p.start, p.k, p.v, p.q = [100], [30], np.array([0, 30]), p.k[:100], p.v[:100], p.q[:30]
        p.check(torch.from_numpy(out[:30]), torch.from_numpy(lse[:30]))

        def only_values(k, v):
            v[100, :, 40:] = np.inf
        p = Problem(kv4, [150], [80], 4, 2, D, 32, dtype, values=only_values)
        out = host(p.run())
        assert np.isfinite(out[:30]).all() and np.isfinite(out[30:, :, :32]).all() and np.isnan(out[30:, :, 32:]).all()


def test_chunks_skip_pages_that_are_not_there(kv4):
    p = Problem(kv4, [160], [60], 4, 2, 128, 32, torch.float32)
    p.table[0, 1], p.table[0, 3] = -5, 10**6
    out, lse = host(p.run()), host(p.lse)
    keep = np.r_[0:32, 64:96, 128:160]
    for i in (0, 31, 59):
        seen = keep[keep <= 100 + i]
        for g in range(2):
            ref, ref_lse, s = orc.attention(host(p.q).astype(np.float64)[i:i + 1, 2 * g:2 * g + 2], p.k[seen, g], p.v[seen, g], 1, p.scale)
            assert np.all(np.abs(out[i:i + 1, 2 * g:2 * g + 2] - ref) <= 5e-5 * s)
            assert np.all(np.abs(lse[i:i + 1, 2 * g:2 * g + 2] - ref_lse) <= 2e-5 + 1e-6 * np.abs(ref_lse))
