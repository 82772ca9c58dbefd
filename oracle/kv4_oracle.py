"""Plain definitions of the paged 4-bit cache and of what runs on it: numpy, 64 bits, one step at a time.

Used by the tests only; shares no code with the library.
"""
from __future__ import annotations

import math

import numpy as np

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
NOT_FINITE = 255
ST_OK, ST_NO_FREE_PAGE, ST_BAD_LENGTH, ST_BAD_TREE = 0, -4, -5, -6


# ---- codes -----------------------------------------------------------------------------------------------

def encode_group(x):
    """(codes [32], scale byte) of the 32 channels of a group."""
    x = [float(v) for v in x]
    if not all(math.isfinite(v) for v in x):
        return [0] * 32, NOT_FINITE
    most = max(abs(v) for v in x)
    e = -126
    while e < 125 and most > 7 * 2.0 ** e:
        e += 1
    codes = []
    for v in x:
        y = abs(v) / 2.0 ** e
        best = min(range(8), key=lambda c: (abs(GRID[c] - y), c % 2))    # ties to the even code
        codes.append(best + (8 if math.copysign(1.0, v) < 0 else 0))
    return codes, e + 127


def decode_group(codes, byte):
    if byte == NOT_FINITE:
        return [math.nan] * 32
    return [(-1 if c & 8 else 1) * GRID[c & 7] * 2.0 ** (byte - 127) for c in codes]


def encode_rows(x):
    """Rows [n, D] as (codes [n, D], scale bytes [n, D / 32]), the same in array form."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(len(x), -1, 32)
    finite = np.isfinite(g).all(axis=-1)
    most = np.where(finite, np.abs(np.where(np.isfinite(g), g, 0)).max(axis=-1), 0)
    e = np.full(most.shape, -126)
    for step in range(-126, 125):
        e = np.where(most > 7 * 2.0 ** step, step + 1, e)
    y = np.abs(np.where(finite[..., None], g, 0)) / (2.0 ** e)[..., None]
    codes = np.zeros(y.shape, dtype=np.int64)
    for c in range(1, 8):
        middle = (GRID[c - 1] + GRID[c]) / 2
        codes += (y >= middle) if c % 2 == 0 else (y > middle)
    codes += 8 * (np.signbit(g) & finite[..., None])
    return codes.reshape(x.shape), np.where(finite, e + 127, NOT_FINITE)


def decode_rows(codes, scales):
    codes = np.asarray(codes)
    grid = np.array(GRID + tuple(-v for v in GRID))
    x = grid[codes].reshape(len(codes), -1, 32)
    factor = np.where(np.asarray(scales) == NOT_FINITE, np.nan, 2.0 ** (np.asarray(scales, dtype=np.float64) - 127))
    return (x * factor[..., None]).reshape(codes.shape)


# ---- pages -----------------------------------------------------------------------------------------------

def page_bytes(page_size, kv_heads, D):
    return kv_heads * page_size * (D // 2 + D // 32) * 2


def _places(page_size, kv_heads, D, slot, head):
    """Byte offsets in a pool of one slot's: key codes, value codes [D / 8 words], key scales, value scales."""
    page, inside = slot // page_size, slot % page_size
    base = page * page_bytes(page_size, kv_heads, D) + (head * (page_size // 32) + inside // 32) * 34 * D
    t = inside % 32
    keys = base + t * (D // 2)
    values = [base + 16 * D + ((t // 4) * (D // 8) + c) * 16 + (t % 4) * 4 for c in range(D // 8)]
    key_scales = base + 32 * D + t * (D // 32)
    value_scales = [base + 33 * D + ((t // 4) * (D // 32) + g) * 4 + t % 4 for g in range(D // 32)]
    return keys, values, key_scales, value_scales


def store(pool, page_size, kv_heads, D, slot, k, v):
    """One token's keys and values [kv_heads, D] into a pool of bytes (in place)."""
    kc, ks = encode_rows(k)
    vc, vs = encode_rows(v)
    for h in range(kv_heads):
        keys, values, key_scales, value_scales = _places(page_size, kv_heads, D, slot, h)
        pool[keys:keys + D // 2] = kc[h, 0::2] + 16 * kc[h, 1::2]
        packed = vc[h, 0::2] + 16 * vc[h, 1::2]
        for c, at in enumerate(values):
            pool[at:at + 4] = packed[4 * c:4 * c + 4]
        pool[key_scales:key_scales + D // 32] = ks[h]
        for g, at in enumerate(value_scales):
            pool[at] = vs[h, g]


def load(pool, page_size, kv_heads, D, slots, head):
    """Keys and values [len(slots), D] of one KV head."""
    kc, vc = np.zeros((2, len(slots), D), dtype=np.int64)
    ks, vs = np.zeros((2, len(slots), D // 32), dtype=np.int64)
    for i, slot in enumerate(slots):
        keys, values, key_scales, value_scales = _places(page_size, kv_heads, D, int(slot), head)
        kb = pool[keys:keys + D // 2].astype(np.int64)
        vb = np.concatenate([pool[at:at + 4] for at in values]).astype(np.int64)
        kc[i, 0::2], kc[i, 1::2] = kb & 15, kb >> 4
        vc[i, 0::2], vc[i, 1::2] = vb & 15, vb >> 4
        ks[i] = pool[key_scales:key_scales + D // 32]
        vs[i] = [pool[at] for at in value_scales]
    return decode_rows(kc, ks), decode_rows(vc, vs)


# ---- page tables -----------------------------------------------------------------------------------------

def _ceil(a, b):
    return -(-a // b)


def pages_plan(page_size, cached, new, free_pages, free_count, table, tokens, pos_start=None, request_tokens=0):
    """The results of a plan as a dict; `table` [R][max_pages] is not changed."""
    R, max_pages = table.shape
    table = table.copy()
    slot_map, token_pos = np.full(tokens, -1), np.full(tokens, -1)
    start, seq_lens, status = [0], [], []
    taken = 0           # pages before this request, of those refused too
    left = free_count
    for r in range(R):
        c, n = int(cached[r]), int(new[r])
        row0 = r * request_tokens if request_tokens else start[-1]
        start.append(start[-1] + max(n, 0))
        ok = c >= 0 and n >= 0 and c + n <= max_pages * page_size and (n == 0 or row0 + n <= tokens) \
            and (request_tokens == 0 or n <= request_tokens)
        need = _ceil(c + n, page_size) - _ceil(c, page_size) if ok else 0
        fits = need == 0 or taken + need <= free_count
        if ok and fits:
            held = _ceil(c, page_size)
            for j in range(need):
                table[r, held + j] = free_pages[free_count - 1 - taken - j]
            left -= need
            for i in range(n):
                page = table[r, (c + i) // page_size]
                slot_map[row0 + i] = page * page_size + (c + i) % page_size if page >= 0 else -1
                token_pos[row0 + i] = (c if pos_start is None else pos_start[r]) + i
        taken += need
        seq_lens.append(c + n if ok and fits else c)
        status.append(ST_BAD_LENGTH if not ok else ST_OK if fits else ST_NO_FREE_PAGE)
    return {"block_table": table, "free_left": left, "seq_lens": np.array(seq_lens), "query_start": np.array(start),
            "slot_map": slot_map, "token_pos": token_pos, "status": np.array(status)}


def pages_release(page_size, finished, seq_lens, table, free_pages, free_count):
    """(seq_lens, table, free_pages, free_count) after the finished requests gave their pages back."""
    seq_lens, table, free_pages = seq_lens.copy(), table.copy(), free_pages.copy()
    back = []
    for r in range(len(seq_lens)):
        if finished[r]:
            back += [page for page in table[r, :_ceil(seq_lens[r], page_size)].tolist() if page >= 0]
            seq_lens[r] = 0
            table[r] = -1
    for i, page in enumerate(reversed(back)):
        free_pages[free_count + i] = page
    return seq_lens, table, free_pages, free_count + len(back)


# ---- norms and rotation ----------------------------------------------------------------------------------

def norm_rope(x, weight, eps, cos, sin, interleaved):
    """One row [D]; cos and sin [rot_dim / 2] of its position."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / math.sqrt(np.mean(x * x) + eps) * np.asarray(weight, dtype=np.float64)
    y, half = x.copy(), len(cos)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[a] = x[a] * cos[i] - x[b] * sin[i]
        y[b] = x[b] * cos[i] + x[a] * sin[i]
    return y


# ---- attention -------------------------------------------------------------------------------------------

def attention(q, k, v, n_new, sm_scale):
    """Queries [n_new, heads, D] of one KV head's group over its keys and values [len, D], causal from the end.
    Returns (out, lse, the weighted sum of |v|, which errors of weights are measured by)."""
    q = np.asarray(q, dtype=np.float64)
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    for i in range(n_new):
        seen = max(len(k) - n_new + i + 1, 0)
        if seen == 0:
            continue
        z = (q[i] @ k[:seen].T) * sm_scale
        top = z.max(axis=1, keepdims=True)
        w = np.exp(z - top)
        total = w.sum(axis=1, keepdims=True)
        out[i] = (w / total) @ v[:seen]
        spread[i] = (w / total) @ np.abs(v[:seen])
        lse[i] = (top + np.log(total))[:, 0]
    return out, lse, spread


# ---- what a token sees -----------------------------------------------------------------------------------

def window_seen(n_keys, n_new, window, sinks):
    """[n_new, n_keys] of truth values: the last `window` keys up to a token's own, and the first `sinks` of those up to its own."""
    seen = np.zeros((n_new, n_keys), dtype=bool)
    for i in range(n_new):
        own = n_keys - n_new + i
        for key in range(min(own + 1, n_keys)):
            seen[i, key] = key > own - window or key < sinks
    return seen


def tree_seen(n_keys, n_new, words, window=0, sinks=0):
    """The same of drafts: words[i] are the words of row i, bit by bit; window 0 is none."""
    seen = np.zeros((n_new, n_keys), dtype=bool)
    base = n_keys - n_new
    for i in range(n_new):
        mine = [j for j in range(n_new) if j // 32 < len(words[i]) and int(words[i][j // 32]) >> (j % 32) & 1]
        own = base + len(mine) - 1
        for key in range(max(base, 0)):
            seen[i, key] = window == 0 or key > own - window or key < sinks
        for j in mine:
            if base + j >= 0:
                seen[i, base + j] = True
    return seen


def seen_attention(q, k, v, seen, sm_scale):
    """`attention` in which query i sees the keys that seen[i] names."""
    q = np.asarray(q, dtype=np.float64)
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    for i in range(len(q)):
        at = np.nonzero(seen[i])[0]
        if not len(at):
            continue
        z = (q[i] @ k[at].T) * sm_scale
        top = z.max(axis=1, keepdims=True)
        w = np.exp(z - top)
        total = w.sum(axis=1, keepdims=True)
        out[i] = (w / total) @ v[at]
        spread[i] = (w / total) @ np.abs(v[at])
        lse[i] = (top + np.log(total))[:, 0]
    return out, lse, spread


# ---- trees of drafts -------------------------------------------------------------------------------------

def _drafts(query_start, r, tokens):
    first, end = (min(max(int(x), 0), tokens) for x in query_start[r:r + 2])
    return first, max(end - first, 0)


def tree_plan(query_start, parents, pos_start, words):
    """(rows of words [T, words], positions [T], status [R])."""
    T = len(parents)
    mask, pos, status = np.zeros((T, words), dtype=np.int64), np.full(T, -1), []
    for r in range(len(query_start) - 1):
        first, n = _drafts(query_start, r, T)
        mine = [int(x) for x in parents[first:first + n]]
        status.append(ST_BAD_LENGTH if n > 32 * words else ST_BAD_TREE if any(a >= i for i, a in enumerate(mine)) else ST_OK)
        if status[-1] != ST_OK:
            continue
        for i in range(n):
            chain = [i]
            while mine[chain[-1]] >= 0:
                chain.append(mine[chain[-1]])
            for j in chain:
                mask[first + i, j // 32] |= 1 << (j % 32)
            at = int(pos_start[r]) + len(chain) - 1
            pos[first + i] = at if at < 2**31 else -1
    return mask, pos, np.array(status)


def tree_keep(query_start, parents, tokens, chosen, cached_lens, max_path, slot_map=None, n_slots=0, status=None):
    """(paths [R, max_path], accepted, next tokens, lengths, moves [(from slot, to slot)] in their order)."""
    T, R = len(parents), len(query_start) - 1
    path, accepted, following, lens, moves = np.full((R, max_path), -1), np.zeros(R, int), np.full(R, -1), np.zeros(R, int), []
    for r in range(R):
        first, n = _drafts(query_start, r, T)
        has_slot = lambda i: slot_map is None or 0 <= slot_map[first + i] < n_slots  # noqa: E731
        kept = [0] if n and has_slot(0) and (status is None or status[r] == ST_OK) else []
        while kept and len(kept) < max_path:
            here = kept[-1]
            want = chosen[first + here]
            children = [c for c in range(here + 1, n) if parents[first + c] == here and tokens[first + c] == want >= 0]
            if not children:
                break
            kept.append(children[0])
        path[r, :len(kept)] = kept
        accepted[r] = len(kept)
        if kept:
            want = chosen[first + kept[-1]]
            following[r] = want if want >= 0 else -1
        lens[r] = cached_lens[r] + len(kept)
        if slot_map is not None:
            moves += [(int(slot_map[first + i]), int(slot_map[first + j])) for j, i in enumerate(kept)
                      if i != j and has_slot(i) and has_slot(j)]
    return path, accepted, following, lens, moves


def move(pool, page_size, kv_heads, D, source, target):
    """The bytes of one slot's row to another slot (in place)."""
    for h in range(kv_heads):
        a, b = _places(page_size, kv_heads, D, source, h), _places(page_size, kv_heads, D, target, h)
        pool[b[0]:b[0] + D // 2] = pool[a[0]:a[0] + D // 2].copy()
        for x, y in zip(a[1], b[1]):
            pool[y:y + 4] = pool[x:x + 4].copy()
        pool[b[2]:b[2] + D // 32] = pool[a[2]:a[2] + D // 32].copy()
        for x, y in zip(a[3], b[3]):
            pool[y] = pool[x]


def pages_trim(page_size, held_lens, seq_lens, table, free_pages, free_count, window=0, sinks=0):
    """(table, free_pages, pages on the stack, pages of each request that went back)."""
    table, free_pages, back, given = table.copy(), free_pages.copy(), [], []
    count = min(max(free_count, 0), len(free_pages))
    for r in range(len(table)):
        most = table.shape[1] * page_size
        held, length, mine = min(max(int(held_lens[r]), 0), most), min(max(int(seq_lens[r]), 0), most), 0
        for j in range(_ceil(held, page_size)):
            tokens = range(j * page_size, (j + 1) * page_size)
            unseen = tokens[0] >= length or (window > 0 and tokens[0] >= sinks and tokens[-1] <= length - window)
            if unseen and table[r, j] >= 0:
                back.append(table[r, j])
                table[r, j] = -1
                mine += 1
        given.append(mine)
    for i, page in enumerate(back):
        if count + len(back) - 1 - i < len(free_pages):
            free_pages[count + len(back) - 1 - i] = page
    return table, free_pages, min(count + len(back), len(free_pages)), np.array(given)
