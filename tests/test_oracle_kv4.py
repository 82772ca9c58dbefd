"""Pins of the paged 4-bit cache's plain definitions (no GPU): hand values, closed forms and second opinions."""
import math

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as orc


def test_group_by_hand():
    x = [0.0] * 32
    x[:8] = [6.0, -6.0, 0.25, 0.75, 1.25, 2.5, -5.0, 3.5]     # scale 1: every middle goes to the even code
    codes, byte = orc.encode_group(x)
    assert byte == 127 and codes[:8] == [7, 15, 0, 2, 2, 4, 14, 6]
    assert orc.decode_group(codes, byte)[:8] == [6.0, -6.0, 0.0, 1.0, 1.0, 2.0, -4.0, 4.0]


def test_scale_holds_up_to_seven_times_it():
    for top, byte in ((7.0, 127), (7.0000001, 128), (3.5, 126), (3.51, 127), (1e-45, 1), (0.0, 1), (3.3e38, 252)):
        x = [top] + [0.0] * 31
        assert orc.encode_group(x)[1] == byte, top


def test_error_is_at_most_half_the_widest_step():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64)) * np.exp(rng.uniform(-20, 20, (200, 1)))
    codes, scales = orc.encode_rows(x)
    step = np.repeat(2.0 ** (scales - 127.0), 32, axis=1)
    assert np.all(np.abs(orc.decode_rows(codes, scales) - x) <= step)


def test_array_form_is_the_group_form():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal((20, 64)), rng.integers(-28, 29, (40, 64)) / 4.0])
    x[3, 5], x[4, 40], x[5, 0], x[6, 1] = math.inf, math.nan, -0.0, -1e-30
    codes, scales = orc.encode_rows(x)
    for r in range(len(x)):
        for g in range(2):
            c, s = orc.encode_group(x[r, 32 * g:32 * g + 32])
            assert codes[r, 32 * g:32 * g + 32].tolist() == c and scales[r, g] == s
            np.testing.assert_array_equal(orc.decode_rows(codes[r:r + 1], scales[r:r + 1])[0, 32 * g:32 * g + 32], orc.decode_group(c, s))


@pytest.mark.parametrize("D", [64, 128])
def test_every_byte_of_a_page_belongs_to_one_token(D):
    heads, page = 3, 64
    used = np.zeros(2 * orc.page_bytes(page, heads, D), dtype=np.int64)
    for slot in range(2 * page):
        for h in range(heads):
            keys, values, key_scales, value_scales = orc._places(page, heads, D, slot, h)
            used[keys:keys + D // 2] += 1
            for at in values:
                used[at:at + 4] += 1
            used[key_scales:key_scales + D // 32] += 1
            used[value_scales] += 1
    assert np.all(used == 1)


def test_what_is_stored_is_loaded():
    rng = np.random.default_rng(2)
    pool = rng.integers(0, 256, 3 * orc.page_bytes(32, 2, 64)).astype(np.uint8)
    k, v = rng.standard_normal((2, 2, 64))
    before = pool.copy()
    orc.store(pool, 32, 2, 64, 45, k, v)
    for h in range(2):
        got_k, got_v = orc.load(pool, 32, 2, 64, [45], h)
        np.testing.assert_array_equal(got_k[0], orc.decode_rows(*orc.encode_rows(k))[h])
        np.testing.assert_array_equal(got_v[0], orc.decode_rows(*orc.encode_rows(v))[h])
    assert np.count_nonzero(before != pool) <= 2 * 2 * (32 + 2)


def test_plan_by_hand():
    table = np.full((3, 4), -1)
    table[0, 0] = 9
    stack = np.array([4, 5, 6, 7, 8])
    p = orc.pages_plan(32, [30, 0, 0], [4, 40, 100], stack, 5, table, 150)
    assert p["block_table"].tolist() == [[9, 8, -1, -1], [7, 6, -1, -1], [-1] * 4]      # the third needs four, two are left
    assert p["status"].tolist() == [0, 0, -4] and p["free_left"] == 2
    assert p["seq_lens"].tolist() == [34, 40, 0] and p["query_start"].tolist() == [0, 4, 44, 144]
    assert p["slot_map"][:6].tolist() == [9 * 32 + 30, 9 * 32 + 31, 8 * 32, 8 * 32 + 1, 7 * 32, 7 * 32 + 1]
    assert p["token_pos"][:6].tolist() == [30, 31, 32, 33, 0, 1] and np.all(p["slot_map"][44:] == -1)


def test_release_undoes_a_plan():
    rng = np.random.default_rng(3)
    stack = rng.permutation(64)
    new = rng.integers(0, 200, 9)
    p = orc.pages_plan(32, np.zeros(9, int), new, stack, 64, np.full((9, 7), -1), int(new.sum()))
    lens, table, free, count = orc.pages_release(32, np.ones(9), p["seq_lens"], p["block_table"], stack, p["free_left"])
    assert count == 64 and not lens.any() and np.all(table == -1)
    np.testing.assert_array_equal(free, stack)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_complex_numbers(interleaved):
    rng = np.random.default_rng(4)
    x, angle = rng.standard_normal(64), rng.uniform(0, 6, 16)
    y = orc.norm_rope(x, None, 0.0, np.cos(angle), np.sin(angle), interleaved)
    a, b = (np.arange(0, 32, 2), np.arange(1, 32, 2)) if interleaved else (np.arange(16), np.arange(16, 32))
    z = (x[a] + 1j * x[b]) * np.exp(1j * angle)
    np.testing.assert_allclose(y[a], z.real, atol=1e-14)
    np.testing.assert_allclose(y[b], z.imag, atol=1e-14)
    np.testing.assert_array_equal(y[32:], x[32:])


def test_norm_gives_unit_mean_square():
    x = np.random.default_rng(5).standard_normal(128) * 7
    y = orc.norm_rope(x, np.full(128, 2.0), 0.0, np.zeros(0), np.zeros(0), False)
    assert abs(np.mean(y * y) - 4.0) < 1e-12


def test_attention_against_scaled_dot_product():
    rng = np.random.default_rng(6)
    q, k, v = rng.standard_normal((5, 3, 64)), rng.standard_normal((20, 64)), rng.standard_normal((20, 64))
    out, lse, _ = orc.attention(q, k, v, 5, 0.3)
    mask = torch.arange(20)[None] <= 15 + torch.arange(5)[:, None]
    t = lambda a: torch.from_numpy(a)  # noqa: E731
    ref = torch.nn.functional.scaled_dot_product_attention(t(q).transpose(0, 1), t(k)[None].expand(3, -1, -1),
                                                           t(v)[None].expand(3, -1, -1), attn_mask=mask, scale=0.3)
    np.testing.assert_allclose(out, ref.transpose(0, 1).numpy(), atol=1e-13)
    z = (t(q) @ t(k).T * 0.3).masked_fill(~mask[:, None], -math.inf)
    np.testing.assert_allclose(lse, torch.logsumexp(z, -1).numpy(), atol=1e-13)


def test_attention_rows_that_see_nothing():
    k, v = np.ones((2, 64)), np.ones((2, 64))
    out, lse, _ = orc.attention(np.ones((4, 1, 64)), k, v, 4, 1.0)
    assert not out[:2].any() and np.all(out[2:] == 1) and np.all(np.isneginf(lse[:2])) and lse[3, 0] == 64 + math.log(2)
