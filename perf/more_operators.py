"""Performance cases of attention over the paged 4-bit cache where a token does not see all that is cached before it, and of
what a serving program calls around it.

Five kinds of call:

  window  kv4.window_attention: single tokens, drafts and chunks of prompts that see the last `window` tokens and the
          first `sinks` ones
  tree    kv4.tree_attention: drafted tokens that form a tree, over what is cached; with a window where the case says so
  plan    kv4.tree_plan: from the drafts' parents the bits of what each of them sees, and its position
  keep    kv4.tree_keep: follows the tokens that the model chose through the tree and moves the rows of those it passes to
          the front.  A pass stores the drafts' rows (kv4.store) as a step does, and reads them back (kv4.load)
  trim    kv4.pages_trim: pages of which no token will be seen again go back onto the free stack.  A pass takes the
          drafts' pages first (kv4.pages_plan) where the case has drafts

The plain forms below compute the same with elementary torch operations in 32 bits.  Inputs are synthetic: normal rows
rounded to the storage type, request lengths spread evenly over the logarithm between the shortest and the longest, pages
handed out in a random order, trees in which every draft's parent is any draft before it.

A page of the cache holds `page` tokens of all KV heads, as [kv_heads][page / 32] blocks of 32 tokens.  A block has
16 D bytes of key codes ([token][D / 2]), 16 D bytes of value codes ([token / 4][D / 8][token % 4][4]), D bytes of key
scales ([token][D / 32]) and D bytes of value scales ([token / 4][D / 32][token % 4]).  A code is a sign and one of
0, 0.5, 1, 1.5, 2, 3, 4, 6, the even channel in the low half of its byte; a scale byte s stands for 2^(s - 127).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
VOCABULARY = 128000


def _case(name, kind, requests, shortest, longest, new_least, new_most, **more):
    case = {"name": name} if name else {}
    case.update(kind=kind, requests=requests, shortest=shortest, longest=longest, new_least=new_least, new_most=new_most)
    case.update({"q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "page": 64, "window": 0, "sinks": 0,
                 "layers": 1, **more})
    return case


def listed():
    return [
        # throughput serving: 64 requests from the first tokens to 32K, of which a layer with a window reads the last 4096
        _case("window_step64", "window", 64, 200, 32768, 1, 1, window=4096, sinks=4),
        # drafts of up to 5 tokens in a row, a window and sinks that end inside a block, single precision, 64 channels
        _case("window_drafts_f32", "window", 24, 60, 4001, 2, 5, window=257, sinks=33, head_dim=64, dtype="f32", page=32),
        # a chunk of a long prompt
        _case("window_chunk32k", "window", 1, 32768, 32768, 2048, 2048, window=4096, sinks=4),
        # interactive generation: a tree of 26 drafts of one sequence over its compressed prompt
        _case("tree_one", "tree", 1, 3277, 3277, 26, 26),
        # generation in a batch of 16 with 16 drafts each
        _case("tree_step16", "tree", 16, 4096, 5120, 16, 16),
        # wide trees over short and long sequences
        _case("tree_wide", "tree", 8, 1000, 16384, 33, 64),
        # the drafts of 16 requests
        _case("plan_step16", "plan", 16, 4096, 5120, 16, 64),
        # chains and trees of 512 requests, from one draft to 256
        _case("plan_many", "plan", 512, 1, 16384, 1, 256),
        # one layer of 16 requests' drafts
        _case("keep_layer", "keep", 16, 4096, 5120, 16, 64),
        # the 32 layers of a model in one pool, single precision
        _case("keep_model_f32", "keep", 16, 200, 4001, 16, 33, layers=32, dtype="f32"),
        # pages that only refused drafts had go back after a step
        _case("trim_step16", "trim", 16, 4096, 5120, 16, 64, page=32),
        # 512 prompts have been processed; of their pages those under a window and the sinks stay
        _case("trim_window512", "trim", 512, 200, 32768, 0, 0, window=1024, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 8), (32, 8), (16, 8), (8, 8), (40, 8), (28, 4), (64, 8), (8, 2), (4, 4)]


def draw(rng: random.Random):
    """One more case of the ranges above: sizes log-uniform, head layouts and options mixed."""
    u, page = rng.random(), rng.choice([32, 64, 64, 128])
    q_heads, kv_heads = rng.choice(HEADS)
    head_dim, dtype = rng.choice([(128, "bf16")] * 4 + [(64, "bf16")] * 2 + [(128, "f32"), (64, "f32")])
    heads = dict(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, page=page)
    seen = dict(window=_log_int(rng, 1, 8192), sinks=rng.choice([0, 4, 4, _log_int(rng, 1, 128)]))
    longest = _log_int(rng, 40, 32768)
    shortest = max(8, longest // _log_int(rng, 1, 100))
    if u < 0.25:
        requests = _log_int(rng, 1, max(1, min(256, (1 << 29) // (longest * kv_heads * head_dim))))
        return _case(None, "window", requests, shortest, longest, 1, rng.choice([1, 1, 1, 4, 8]), **heads, **seen)
    if u < 0.4:
        longest = _log_int(rng, 200, 16384)
        new = _log_int(rng, 30, min(longest, 2048))
        keys = min(longest, seen["window"] + seen["sinks"] + new)
        requests = _log_int(rng, 1, max(1, min(16, (1 << 28) // (keys * new * q_heads))))
        return _case(None, "window", requests, longest // rng.choice([1, 2]), longest, max(1, new // rng.choice([1, 3])), new,
                     **heads, **seen)
    drafts = _log_int(rng, 2, 96)
    if u < 0.7:
        drafts = min(drafts, longest)
        requests = _log_int(rng, 1, max(1, min(32, (1 << 28) // (longest * max(drafts * q_heads, 8 * head_dim)))))
        return _case(None, "tree", requests, shortest, longest, max(1, drafts // rng.choice([1, 3])), drafts, **heads,
                     **(seen if rng.random() < 0.3 else {}))
    requests = _log_int(rng, 1, 512)
    if u < 0.8:
        return _case(None, "plan", requests, shortest, longest, 1, _log_int(rng, 2, 256))
    if u < 0.9:
        requests, layers = min(requests, 32), rng.choice([1, 1, 8, 32])
        while requests * drafts * layers * kv_heads * head_dim > 1 << 26:
            requests, drafts = max(1, requests // 2), max(2, drafts // 2)
        return _case(None, "keep", requests, shortest, longest, max(1, drafts // 2), drafts, layers=layers, **heads)
    if rng.random() < 0.5:
        return _case(None, "trim", requests, shortest, longest, max(1, drafts // 2), drafts, page=page)
    return _case(None, "trim", requests, shortest, longest, rng.choice([0, 1]), rng.choice([1, drafts]), page=page, **seen)


# ---- inputs ----------------------------------------------------------------------------------------------

def _spread(n, least, most):
    """n whole numbers, evenly spread over the logarithm between least and most (least where that is 0)."""
    if least < 1:
        return np.full(n, least, dtype=np.int64)
    at = (np.arange(n) + 0.5) / n if n > 1 else np.ones(1)
    return np.rint(least * (most / least) ** at).astype(np.int64)


def _lengths(case):
    """(tokens of each request with its new ones, new tokens of each): what `work` counts, in no order."""
    total, new = _spread(case["requests"], case["shortest"], case["longest"]), _spread(case["requests"], case["new_least"], case["new_most"])
    return total, np.minimum(new, total)


def _page_bytes(case):
    return case["kv_heads"] * case["page"] * case["head_dim"] * 34 // 32


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _i32(a):
    return _dev(np.asarray(a).astype(np.int32))


def _fill_pages(case, n_pages, gen):
    """A pool whose every row holds the 4-bit codes of normal keys and values."""
    D, H, blocks = case["head_dim"], case["kv_heads"], case["page"] // 32
    pages = torch.zeros((n_pages, _page_bytes(case)), dtype=torch.uint8, device="cuda")
    for part in pages.split(max(1, (1 << 27) // (H * case["page"] * D))):
        rows = torch.randn((2, len(part), H, blocks, 32, D), generator=gen, device="cuda")
        views = _views(part, case)
        codes, scales = _quantise(rows)
        for i, name in enumerate("kv"):
            views[name].copy_(codes[i].unflatten(-2, views[name].shape[-3:-1]) if name == "v" else codes[i])
            views[name + "s"].copy_(scales[i].unflatten(-2, views[name + "s"].shape[-3:-1]) if name == "v" else scales[i])
    return pages


def _tables(need, spare, rng, columns):
    """A block table with pages in a random order, and the pages that are left."""
    pool = rng.permutation(int(need.sum()) + spare)
    table = np.full((len(need), columns), -1)
    listed_ = np.arange(columns)[None, :] < need[:, None]
    table[listed_] = pool[:int(need.sum())]
    return table, pool[int(need.sum()):]


def _trees(new, rng):
    """Parents of all drafts: -1 for the first of a request, any earlier one for the others."""
    index = np.arange(int(new.sum())) - np.repeat(np.cumsum(new) - new, new)
    return np.where(index == 0, -1, np.floor(rng.random(len(index)) * index)).astype(np.int64), index


def _masks(parents, index, words):
    """Bit j of row i: draft j of its request is i or an ancestor of it."""
    rows = np.zeros((len(parents), words), dtype=np.uint32)
    for t, (parent, i) in enumerate(zip(parents.tolist(), index.tolist())):
        if parent >= 0:
            rows[t] = rows[t - i + parent]
        rows[t, i // 32] |= np.uint32(1 << (i % 32))
    return rows.view(np.int32)


def _prepare_attention(case, gen, rng):
    R, H, D, B, dtype = case["requests"], case["q_heads"], case["head_dim"], case["page"], DTYPES[case["dtype"]]
    lens, new = _lengths(case)
    order = rng.permutation(R)
    lens, new = lens[order], new[order]
    need = -(-lens // B)
    table, _ = _tables(need, 1, rng, int(need.max()))
    T, most = int(new.sum()), int(new.max())
    q = torch.empty((T, H, D), dtype=dtype, device="cuda")
    q.copy_(2 * torch.randn(q.shape, generator=gen, device="cuda"))
    s = {"q": q, "pages": _fill_pages(case, int(need.sum()) + 1, gen), "table": _i32(table), "lens": _i32(lens),
         "start": _i32(np.concatenate([[0], np.cumsum(new)])), "most": most, "out": torch.zeros_like(q),
         "lse": torch.zeros((T, H), dtype=torch.float32, device="cuda")}
    if case["kind"] == "tree":
        s["mask"] = _dev(_masks(*_trees(new, rng), -(-most // 32)))
    return s


def _prepare_tree(case, gen, rng):
    """Drafts of requests: parents, tokens and what the model chose after each, mostly one of its children."""
    R, B = case["requests"], case["page"]
    lens, new = _lengths(case)
    order = rng.permutation(R)
    lens, new = lens[order], new[order]
    T, most = int(new.sum()), int(new.max())
    parents, index = _trees(new, rng)
    tokens, chosen = rng.integers(0, VOCABULARY, T), rng.integers(0, VOCABULARY, T)
    child = np.nonzero((parents >= 0) & (rng.random(T) < 0.8))[0]
    chosen[(child - index[child]) + parents[child]] = tokens[child]
    s = {"parents": _i32(parents), "start": _i32(np.concatenate([[0], np.cumsum(new)])), "most": most,
         "base": _i32(lens - new), "tokens": _i32(tokens), "chosen": _i32(chosen), "lens": _i32(lens)}
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    if case["kind"] == "plan":
        s["out"] = {"tree_mask": zeros(T, -(-most // 32)), "token_pos": zeros(T), "status": zeros(R)}
        return s
    # the places of the drafts, which come after what a request holds; a layer has its pages behind those of the one before it
    need, L = -(-lens // B) - (lens - new) // B, case["layers"]
    table, _ = _tables(need, 0, rng, int(need.max()))
    at = np.repeat((lens - new) % B, new) + index
    slots = table[np.repeat(np.arange(R), new), at // B] * B + at % B
    layer = int(need.sum())
    s["slots"] = _i32(slots)
    s["all_slots"] = _i32((np.arange(L)[:, None] * layer * B + slots[None, :]).reshape(-1))
    dtype, shape = DTYPES[case["dtype"]], (L * T, case["kv_heads"], case["head_dim"])
    s["pages"] = _fill_pages(case, L * layer, gen)
    for name in ("k", "v"):
        s[name] = torch.randn(shape, generator=gen, device="cuda").to(dtype)
        s[name + "_values"] = torch.zeros(shape, dtype=dtype, device="cuda")
    s["out"] = {"path": zeros(R, most), "accepted": zeros(R), "next_token": zeros(R), "seq_lens": zeros(R)}
    return s


def _prepare_trim(case, gen, rng):
    """Requests before a step; `kept` tokens are theirs after it: one at least of the drafts."""
    R, B = case["requests"], case["page"]
    lens, new = _lengths(case)
    order = rng.permutation(R)
    lens, new = lens[order], new[order]
    base = lens - new
    kept = base + np.minimum(new, rng.integers(1, 9, R))
    held, need = -(-base // B), -(-lens // B)
    table, spare = _tables(held, int((need - held).sum()) + R, rng, int(need.max()) + 1)
    R, columns = table.shape
    T = int(new.sum())
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    # the table and the stack in one array, which a pass starts from as they were
    before = _i32(np.concatenate([table.reshape(-1), spare, np.full(int(held.sum()), -1)]))
    both = before.clone()
    return {"before": before, "both": both, "table": both[:R * columns].view(R, columns), "free": both[R * columns:],
            "count": _i32([len(spare)]), "base": _i32(base), "new": _i32(new), "lens": _i32(lens), "kept": _i32(kept), "T": T,
            "plan": {"free_left": zeros(1), "seq_lens": zeros(R), "query_start": zeros(R + 1), "slot_map": zeros(T),
                     "token_pos": zeros(T), "status": zeros(R)},
            "free_left": zeros(1), "given_back": zeros(R)}


def prepare(case, seed):
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    make = {"window": _prepare_attention, "tree": _prepare_attention, "plan": _prepare_tree, "keep": _prepare_tree,
            "trim": _prepare_trim}
    return {"case": case, **make[case["kind"]](case, gen, rng)}


# ---- the 4-bit cache in plain torch ----------------------------------------------------------------------

def _quantise(x):
    """Rows [..., D] as (codes [..., D / 2], scale bytes [..., D / 32])."""
    x = x.float().unflatten(-1, (-1, 32))
    most = x.abs().amax(dim=-1, keepdim=True)
    part, power = torch.frexp(most)                                 # most = part * 2^power, part in [0.5, 1)
    e = torch.where(part <= 0.875, power - 3, power - 2).clamp(-126, 125)   # least e with most <= 7 * 2^e
    e = torch.where(most > 0, e, -126)
    y = torch.ldexp(x.abs(), -e)
    code = ((y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)
            + 8 * torch.signbit(x).byte()).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).byte().squeeze(-1)


def _dequantise(codes, scales):
    """Rows [..., D] in 32 bits of codes [..., D / 2] and scale bytes [..., D / 32]."""
    one = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    two = torch.stack([one.repeat(16), one.repeat_interleave(16)], dim=1)     # the two values of a byte
    x = two[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    return (x * torch.exp2(scales.float() - 127)[..., None]).flatten(-2)


def _views(pages, case):
    """Codes and scales in a pool of pages [n][page bytes]: of keys [n][kv_heads][page / 32][32][...], of values by fours of
    tokens, [n][kv_heads][page / 32][8][4][...]."""
    D = case["head_dim"]
    block = pages.view(len(pages), case["kv_heads"], case["page"] // 32, 34 * D)
    values = block[..., 16 * D:32 * D].unflatten(-1, (8, D // 8, 4, 4)).transpose(-3, -2)     # [8][4 tokens][D / 8][4 bytes]
    return {"k": block[..., :16 * D].unflatten(-1, (32, D // 2)), "ks": block[..., 32 * D:33 * D].unflatten(-1, (32, D // 32)),
            "v": _Pieces(values), "vs": block[..., 33 * D:].unflatten(-1, (8, D // 32, 4)).transpose(-2, -1)}


class _Pieces:
    """Codes of values [..., 8, 4, D / 8, 4], seen as [..., 8, 4, D / 2]."""

    def __init__(self, t):
        self.t, self.shape = t, t.shape[:-2] + (t.shape[-2] * t.shape[-1],)

    def copy_(self, rows):
        self.t.copy_(rows.unflatten(-1, self.t.shape[-2:]))

    def __getitem__(self, at):
        return self.t[at].flatten(-2)

    def __setitem__(self, at, rows):
        self.t[at] = rows.unflatten(-1, self.t.shape[-2:])


def _at(slots, case):
    """Where slots are, of keys and of values: page, every KV head, block, token."""
    slots = slots.long()
    page, block, token = slots // case["page"], slots % case["page"] // 32, slots % 32
    return (page, slice(None), block, token), (page, slice(None), block, token // 4, token % 4)


def _rows_of(case, pages, slots):
    """Keys and values [len(slots), kv_heads, D] in 32 bits."""
    keys, values = _at(slots, case)
    views = _views(pages, case)
    return _dequantise(views["k"][keys], views["ks"][keys]), _dequantise(views["v"][values], views["vs"][values])


def _put_rows(case, pages, slots, k, v):
    keys, values = _at(slots, case)
    views = _views(pages, case)
    views["k"][keys], views["ks"][keys] = _quantise(k)
    views["v"][values], views["vs"][values] = _quantise(v)


# ---- the operators in plain torch ------------------------------------------------------------------------

def _plain_attention(s, case):
    """Attention over the keys that a request's window, sinks and drafts can reach, the others are not looked at."""
    q, table, lens, start, most = s["q"], s["table"], s["lens"].long(), s["start"].long(), s["most"]
    R, H, Hkv, D, B = case["requests"], case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    G, dev, tree = H // Hkv, q.device, case["kind"] == "tree"
    sinks, window = case["sinks"], case["window"] or 1 << 30
    new = start[1:] - start[:-1]
    base = lens - new
    index = torch.arange(most, device=dev)
    token = torch.arange(len(q), device=dev)
    request = torch.searchsorted(start, token, right=True) - 1
    own_index = token - start[request]
    padded = torch.zeros((R, most, H, D), device=dev)
    padded[request, own_index] = q.float()
    # positions of the keys: the sinks, and what comes after the first key in any window
    if tree:
        bits = (s["mask"][:, index // 32] >> (index % 32)) & 1
        sees = torch.zeros((R, most, most), dtype=torch.bool, device=dev)
        sees[request, own_index] = (bits == 1) & (index < new[request, None])
        place = base[:, None] - 1 + sees.sum(dim=-1)        # the position of a draft is as deep as it has ancestors
        reach = min(window, int(case["longest"])) + most
    else:
        place = base[:, None] + index
        reach = min(window, int(case["longest"])) + most - 1
    first = (lens - reach).clamp(min=0)
    key = first[:, None] + torch.arange(min(reach, int(case["longest"])), device=dev)
    sink = torch.arange(sinks, device=dev).expand(R, sinks)
    key = torch.cat([torch.where(sink < first[:, None], sink, 1 << 30), key], dim=1)
    there = key < lens[:, None]
    at = torch.where(there, key, 0)
    slots = table.long().gather(1, at // B) * B + at % B
    k, v = _rows_of(case, s["pages"], slots.flatten())
    key, there = key[:, None, :], there[:, None, :]
    visible = there & ((key > place[:, :, None] - window) | (key < sinks))
    if tree:
        draft = (key - base[:, None, None]).expand(R, most, key.shape[-1])
        visible = torch.where(draft < 0, visible, there & sees.gather(2, draft.clamp(0, most - 1)))
    else:
        visible = visible & (key <= place[:, :, None])
    rows = lambda x: x.view(R, -1, Hkv, D).transpose(1, 2).contiguous()  # noqa: E731
    z = padded.view(R, most, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, G * most, D)
    z = torch.matmul(z, rows(k).transpose(2, 3)).view(R, Hkv, G, most, -1)
    z = z.mul_(1 / math.sqrt(D)).masked_fill_(~visible[:, None, None], -math.inf)
    top = z.amax(dim=-1, keepdim=True).clamp(min=-1e30)
    z = z.sub_(top).exp_()
    total = z.sum(dim=-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    out = torch.matmul(z.view(R, Hkv, G * most, -1), rows(v)).view(R, Hkv, G, most, D) / torch.where(total > 0, total, 1.0)
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).reshape(R, most, H, D)[request, own_index])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(R, most, H)[request, own_index])
    return {"out": s["out"], "lse": s["lse"]}


def _ancestors(s):
    """[R, most, most] of 0 and 1: draft j is i or an ancestor of i.  Also the request and index of every draft, and the padded
    parents (-1 where there is no draft)."""
    start, parents, most = s["start"].long(), s["parents"].long(), s["most"]
    R, dev = len(start) - 1, parents.device
    token = torch.arange(len(parents), device=dev)
    request = torch.searchsorted(start, token, right=True) - 1
    index = token - start[request]
    padded = torch.full((R, most), -1, dtype=torch.int64, device=dev)
    padded[request, index] = parents
    number = torch.arange(most, device=dev)
    up = (number[None, :, None] == number) | (padded[:, :, None] == number)
    up = up.float()
    for _ in range(max(1, (most - 1).bit_length())):        # paths of twice the length each time
        up = torch.matmul(up, up).clamp(max=1)
    return up, request, index, padded


def _plain_plan(s):
    up, request, index, _ = _ancestors(s)
    R, most, o = len(up), s["most"], s["out"]
    words = o["tree_mask"].shape[1]
    bits = torch.zeros((R, most, 32 * words), dtype=torch.int64, device=up.device)
    bits[:, :, :most] = up.long()
    power = torch.ones(32, dtype=torch.int64, device=up.device) << torch.arange(32, device=up.device)
    mask = (bits.unflatten(-1, (words, 32)) * power).sum(dim=-1)
    mask = torch.where(mask >= 1 << 31, mask - (1 << 32), mask)
    o["tree_mask"].copy_(mask[request, index])
    o["token_pos"].copy_(s["base"][request] + up.sum(dim=-1).long()[request, index] - 1)
    o["status"].zero_()
    return dict(o)


def _plain_keep(s, case):
    _put_rows(case, s["pages"], s["all_slots"], s["k"], s["v"])
    up, request, index, parents = _ancestors(s)
    R, most, o, dev = len(up), s["most"], s["out"], up.device
    pad = lambda x: torch.full((R, most), -1, dtype=torch.int64, device=dev).index_put_((request, index), x.long())  # noqa: E731
    tokens, chosen = pad(s["tokens"]), pad(s["chosen"])
    number = torch.arange(most, device=dev)
    there = number < (s["start"][1:] - s["start"][:-1])[:, None]
    wanted = tokens == chosen.gather(1, parents.clamp(min=0))
    twin = (parents[:, :, None] == parents[:, None, :]) & (tokens[:, :, None] == tokens[:, None, :]) & (number < number[:, None])
    fits = (wanted & (parents >= 0) & ~twin.any(dim=-1)) | (number == 0)      # chosen by its parent, the first of its kind
    passed = (torch.matmul(up, (~fits).float()[:, :, None]).squeeze(-1) == 0) & there
    accepted = passed.sum(dim=-1)
    path = torch.where(passed, number, most).sort(dim=-1).values
    last = path.gather(1, (accepted - 1).clamp(min=0)[:, None])
    o["path"].copy_(torch.where(path < most, path, -1))
    o["accepted"].copy_(accepted)
    o["next_token"].copy_(chosen.gather(1, last.clamp(max=most - 1)).squeeze(1))
    o["seq_lens"].copy_(s["base"] + accepted)
    # row path[j] of a request to place j, in every layer
    L, T = case["layers"], len(request)
    source = s["start"].long()[request] + o["path"].long()[request, index]
    source = torch.where(index < accepted[request], source, torch.arange(T, device=dev))
    moved = (torch.arange(L, device=dev)[:, None] * T + source).flatten()
    slots = s["all_slots"].long()
    (keys, values), (from_keys, from_values) = _at(slots, case), _at(slots[moved], case)
    views = _views(s["pages"], case)
    views["k"][keys], views["ks"][keys] = views["k"][from_keys], views["ks"][from_keys]
    views["v"][values], views["vs"][values] = views["v"][from_values], views["vs"][from_values]
    k, v = _rows_of(case, s["pages"], slots)
    s["k_values"].copy_(k)
    s["v_values"].copy_(v)
    return {**o, "k_values": s["k_values"], "v_values": s["v_values"]}


def _plain_trim(s, case):
    B, window, sinks = case["page"], case["window"] or 1 << 30, case["sinks"]
    s["both"].copy_(s["before"])
    table, free, base, lens, kept, count = s["table"], s["free"], s["base"].long(), s["lens"].long(), s["kept"].long(), s["count"]
    page = torch.arange(table.shape[1], device=table.device)[None, :]
    if case["new_most"]:        # pages for the drafts
        held, need = (base + B - 1) // B, (lens + B - 1) // B
        until = (need - held).cumsum(0)
        taken = count - 1 - ((until - (need - held) - held)[:, None] + page)
        given = (page >= held[:, None]) & (page < need[:, None])
        table.copy_(torch.where(given, free[taken.clamp(0, len(free) - 1)], table))
        count = count - until[-1]
    # pages of a request that no token to come sees: behind its end, or between the sinks and the next token's window
    listed_ = page < ((lens + B - 1) // B)[:, None]
    gone = (page * B >= kept[:, None]) | ((page * B >= sinks) & ((page + 1) * B <= kept[:, None] - window + 1))
    back = listed_ & gone & (table >= 0)
    order = back.flatten().cumsum(0)
    to = count + order[-1] - order
    stack = torch.cat([free, free[:1]])         # one more place, for the entries that stay
    stack[torch.where(back.flatten(), to, len(free))] = table.flatten()
    free.copy_(stack[:-1])
    table.masked_fill_(back, -1)
    s["given_back"].copy_(back.sum(dim=1))
    s["free_left"].copy_(count + order[-1])
    return {"table": table, "free": free, "free_left": s["free_left"], "given_back": s["given_back"]}


def _plain(s):
    case = s["case"]
    if case["kind"] == "plan":
        return _plain_plan(s)
    return {"keep": _plain_keep, "trim": _plain_trim}.get(case["kind"], _plain_attention)(s, case)


# ---- the framework's operators ---------------------------------------------------------------------------

def _handles(s):
    """What a program keeps beside its tensors: the cache, the workspace of the attention, the results' arrays."""
    from paper_2502_01941_amd import kv4
    case = s["case"]
    h, o = {"kv4": kv4}, s.get("out")
    if "pages" in s:
        h["cache"] = kv4.Cache(s["pages"], case["page"], case["kv_heads"], case["head_dim"])
    if case["kind"] == "window":
        h["workspace"] = kv4.window_attention_workspace(h["cache"], s["q"], s["table"], case["window"], case["sinks"], s["most"])
    if case["kind"] == "tree":
        h["workspace"] = kv4.tree_attention_workspace(h["cache"], s["q"], s["table"], s["most"], case["window"] or None, case["sinks"])
    if case["kind"] == "plan":
        h["plan"] = kv4.TreePlan(o["tree_mask"], o["token_pos"], o["status"])
    if case["kind"] == "keep":
        h["kept"] = kv4.TreeKept(o["path"], o["accepted"], o["next_token"], o["seq_lens"])
    if case["kind"] == "trim":
        h["plan"] = kv4.PagePlan(s["table"], **s["plan"])
    return h


def _own(s):
    if "handles" not in s:
        s["handles"] = _handles(s)
    h, case = s["handles"], s["case"]
    kv4, kind = h["kv4"], case["kind"]
    if kind == "window":
        kv4.window_attention(h["cache"], s["q"], s["table"], s["lens"], 1 / math.sqrt(case["head_dim"]), case["window"],
                             case["sinks"], s["start"], s["most"], s["out"], s["lse"], h["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "tree":
        kv4.tree_attention(h["cache"], s["q"], s["table"], s["lens"], 1 / math.sqrt(case["head_dim"]), s["start"], s["mask"],
                           s["most"], case["window"] or None, case["sinks"], s["out"], s["lse"], h["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "plan":
        kv4.tree_plan(s["start"], s["parents"], s["base"], h["plan"])
        return dict(s["out"])
    if kind == "keep":
        kv4.store(h["cache"], s["k"], s["v"], s["all_slots"])
        kv4.tree_keep(s["start"], s["parents"], s["tokens"], s["chosen"], s["base"], h["kept"], h["cache"], s["slots"], case["layers"])
        kv4.load(h["cache"], s["all_slots"], s["k_values"], s["v_values"])
        return {**s["out"], "k_values": s["k_values"], "v_values": s["v_values"]}
    s["both"].copy_(s["before"])
    count = s["count"]
    if case["new_most"]:
        kv4.pages_plan(case["page"], s["base"], s["new"], s["free"], count, h["plan"])
        count = s["plan"]["free_left"]
    kv4.pages_trim(case["page"], s["lens"], s["kept"], s["table"], s["free"], count, s["free_left"], s["given_back"],
                   case["window"] or None, case["sinks"])
    return {"table": s["table"], "free": s["free"], "free_left": s["free_left"], "given_back": s["given_back"]}


def run(state):
    return (_own if own else _plain)(state)


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    kind, R, B = case["kind"], case["requests"], case["page"]
    lens, new = _lengths(case)
    size, D, Hkv = 2 if case["dtype"] == "bf16" else 4, case["head_dim"], case["kv_heads"]
    if kind in ("window", "tree"):
        base, window, sinks = lens - new, case["window"] or 1 << 30, case["sinks"]
        first = np.maximum(base - window + 1, 0)        # in the window of the first new token
        extra = np.minimum(first, sinks)                # sinks before it
        keys = (lens - first + extra).sum()
        # keys that the new tokens see in the window, and beside them the sinks; a draft some ancestors and itself
        seen = np.minimum(base, window - 1) + extra
        if kind == "tree":
            pairs = float((new * (seen + np.log2(new + 1))).sum())
        else:
            grow = np.clip(np.minimum(window, lens) - np.minimum(window, base + 1), 0, None)    # tokens until the window is full
            pairs = float((new * (seen + 1) + grow * new - grow * (grow + 1) / 2).sum())
        mask = 4 * int(new.sum()) * (-(-int(new.max()) // 32)) if kind == "tree" else 0
        return {"bytes": float(keys) * Hkv * D * 2 * 17 / 32 + int(new.sum()) * case["q_heads"] * (2 * D * size + 4) + mask,
                "flops": 4.0 * pairs * case["q_heads"] * D}
    T, words = int(new.sum()), -(-int(new.max()) // 32) if new.max() else 1
    if kind == "plan":      # a parent in, a position and its words out; a start and position in and a status out per request
        return {"bytes": 4.0 * (T * (2 + words) + 3 * R), "flops": 0}
    if kind == "keep":      # rows in, and out again; parent, token, chosen and slots; a path out
        rows = case["layers"] * T * Hkv * D
        return {"bytes": 4.0 * rows * size + 4.0 * (4 * T + case["layers"] * T + R * int(new.max()) + 5 * R), "flops": 0}
    # the words of the table and of the stack out; three lengths in and one number out per request; slots and positions of drafts
    return {"bytes": 4.0 * (2 * int((-(-lens // B)).sum()) + 4 * R + 2 * T), "flops": 0}


# ---- the same in 64 bits ---------------------------------------------------------------------------------

def _exact_cached(s, case, r, g):
    """Keys and values of one request and KV head, from the bytes of its pages."""
    D, B, n = case["head_dim"], case["page"], int(s["lens"][r])
    pages = s["table"][r, :-(-n // B)].long()
    size = B * D * 34 // 32
    block = s["pages"][pages][:, g * size:(g + 1) * size].reshape(-1, 34 * D)
    value = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64, device="cuda")

    def of(codes, scales):
        x = torch.stack([value[(codes & 15).long()], value[(codes >> 4).long()]], dim=-1).reshape(len(codes), D // 32, 32)
        return (x * torch.exp2(scales.double() - 127)[..., None]).reshape(len(codes), D)[:n]

    k = of(block[:, :16 * D].reshape(-1, D // 2), block[:, 32 * D:33 * D].reshape(-1, D // 32))
    v = of(block[:, 16 * D:32 * D].reshape(-1, D // 8, 4, 4).transpose(1, 2).reshape(-1, D // 2),
           block[:, 33 * D:].reshape(-1, D // 32, 4).transpose(1, 2).reshape(-1, D // 32))
    return k, v


def _exact_seen(s, case, r):
    """Which of its keys the new tokens of a request see, one row each."""
    start, n_keys = s["start"].tolist(), int(s["lens"][r])
    n = start[r + 1] - start[r]
    base, window, sinks = n_keys - n, case["window"] or 1 << 30, case["sinks"]
    seen = np.zeros((n, n_keys), dtype=bool)
    words = s["mask"][start[r]:start[r + 1]].cpu().numpy().view(np.uint32) if case["kind"] == "tree" else None
    for i in range(n):
        if words is None:
            mine = list(range(i + 1))
            position = base + i
        else:
            mine = [j for j in range(n) if int(words[i, j // 32]) >> (j % 32) & 1]
            position = base + len(mine) - 1
        seen[i, max(position - window + 1, 0):base] = True
        seen[i, :min(sinks, base)] = True
        if words is None:
            mine = [j for j in mine if base + j > position - window or base + j < sinks]
        seen[i, [base + j for j in mine]] = True
    return torch.from_numpy(seen).to("cuda")


def _exact_attention(case, seed):
    s = prepare(case, seed)
    G, D = case["q_heads"] // case["kv_heads"], case["head_dim"]
    start = s["start"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for r in range(case["requests"]):
        seen = _exact_seen(s, case, r)
        mine = slice(start[r], start[r + 1])
        for g in range(case["kv_heads"]):
            k, v = _exact_cached(s, case, r, g)
            for h in range(g * G, (g + 1) * G):
                z = (s["q"][mine, h].double() @ k.T) / math.sqrt(D)
                z = torch.where(seen, z, -math.inf)
                out[mine, h] = torch.softmax(z, dim=-1) @ v
                lse[mine, h] = torch.logsumexp(z, dim=-1)
    return {"out": out, "lse": lse}


def _exact_row_values(x):
    """Rows [..., D] as the cache would hold them, straight from the definition: the nearest multiple of 2^e on the grid."""
    x = x.double().unflatten(-1, (-1, 32))
    most = x.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(most / 7) - 1e-13).clamp(-126, 125)
    y = x.abs() / torch.exp2(e)
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0)).double()
    return (torch.sign(x) * torch.clamp(torch.round(y / step) * step, max=6.0) * torch.exp2(e)).flatten(-2)


def _exact_keep(case, seed):
    s = prepare(case, seed)
    start, parents, tokens, chosen = (s[x].tolist() for x in ("start", "parents", "tokens", "chosen"))
    T, source = len(parents), list(range(len(parents)))
    for first, end in zip(start, start[1:]):
        here, place = first, first
        while True:
            source[place] = here
            place += 1
            children = [t for t in range(here + 1, end) if parents[t] == here - first and tokens[t] == chosen[here]]
            if not children:
                break
            here = children[0]
    at = (np.arange(case["layers"])[:, None] * T + np.array(source)).reshape(-1)
    rows = lambda x: _exact_row_values(x)[_dev(at)]  # noqa: E731
    return {"path": None, "accepted": None, "next_token": None, "seq_lens": None, "k_values": rows(s["k"]), "v_values": rows(s["v"])}


def exact(case, seed):
    if case["kind"] in ("plan", "trim"):
        return None
    return (_exact_keep if case["kind"] == "keep" else _exact_attention)(case, seed)
