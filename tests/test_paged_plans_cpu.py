"""Workspaces of the attention over pages of 8 bits and behind shared prefixes: what a call needs is what its query promised,
for any batch, length and grouping up to what was asked for; and lengths that positions of 32 bits do not reach."""
import ctypes
import random
import re

import pytest

from paper_2401_09670_amd import binding

P = 4096  # an aligned address that nobody follows
INVALID, WORKSPACE = 1, 3
SHAPES = [(256, 4, 64, 0), (5120, 40, 128, 0), (8192, 64, 128, 8), (2048, 16, 128, 1), (4096, 64, 64, 2)]
CACHE = (P, P, P, P, 1 << 20)


def _need(ctx, status):
    """Bytes that a call given no workspace asked for (it is refused before it touches a device)."""
    assert status == WORKSPACE
    text = ctx.lib.ds_last_error(ctx.handle).decode()
    return int(re.search(r"workspace 0 < (\d+)", text).group(1))


@pytest.mark.parametrize("hidden,n,s,n_kv", SHAPES)
def test_a_call_needs_no_more_than_was_promised(hidden, n, s, n_kv):
    ctx = binding.Context(hidden, n, s, 1024, n_kv_heads=n_kv)
    rng, asked, ctx_items = random.Random(hidden), 0, (n_kv or n)
    for _ in range(300):
        B = int(2 ** rng.uniform(0, 8.5))
        L, X = int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 16))
        most_B, most_L, most_X = B + rng.randrange(B + 1), L + rng.randrange(L + 1), X + rng.randrange(X + 1)
        groups = rng.randint(1, B)
        rows = rng.randint(-(-B // groups), B)
        kind = rng.randrange(3)
        scales = (None, None) if kind == 0 else (P, P)
        cache = (P, P, *scales, 1 << 20, kind)
        st = ctx.lib.ds_decode_attention_shared(ctx.handle, P, P, groups, rows, P, P, -(-X // 16), X, P, P, B, -(-L // 16), L,
                                                *cache, P, None, 0, None)
        assert _need(ctx, st) <= ctx.ds_decode_shared_workspace_bytes(most_B, most_X, most_L)
        # 96 pages and few rows are split, whatever else a plan says
        if kind and L >= 1536 and B * ctx_items <= 64:
            asked += 1
            st = ctx.lib.ds_decode_attention_quant(ctx.handle, P, P, P, B, -(-L // 16), L, *cache, P, None, 0, None)
            assert _need(ctx, st) <= ctx.ds_decode_quant_workspace_bytes(most_B, most_L)
    assert asked >= 5
    ctx.close()


@pytest.mark.parametrize("longest", [2 ** 31 - 1, 2 ** 31 - 16])
def test_lengths_that_no_position_reaches(longest):
    ctx = binding.Context(1024, 8, 128, 1024, n_kv_heads=2)
    pages = 2 ** 27
    w = binding.LayerWeights()
    for name, _ in binding.LayerWeights._fields_:
        setattr(w, name, P)
    w, end, cache = ctypes.byref(w), (P, 1 << 40, None), (*CACHE, 1)
    lib, h = ctx.lib, ctx.handle
    assert lib.ds_decode_attention_quant(h, P, P, P, 4, pages, longest, *cache, P, *end) == INVALID
    assert lib.ds_decode_step_quant(h, w, P, P, P, 4, pages, longest, *cache, 2 * P, *end) == INVALID
    for X, Xp, L, Lp in ((longest, pages, 32, 2), (32, 2, longest, pages)):
        assert lib.ds_decode_attention_shared(h, P, P, 2, 3, P, P, Xp, X, P, P, 4, Lp, L, *cache, P, *end) == INVALID
        assert lib.ds_decode_step_shared(h, w, P, P, 2, 3, P, P, Xp, X, P, P, 4, Lp, L, *cache, 2 * P, *end) == INVALID
    ctx.close()


def test_queries_of_the_largest_sizes_return():
    ctx = binding.Context(256, 4, 64, 1024)
    most = 2 ** 31 - 1
    assert ctx.ds_decode_quant_workspace_bytes(4, most) == 0
    assert ctx.ds_decode_shared_workspace_bytes(4, most, 16) == ctx.ds_decode_shared_workspace_bytes(4, 16, most) == 0
    assert 0 < ctx.ds_decode_quant_workspace_bytes(4, 2 ** 30) <= ctx.ds_decode_shared_workspace_bytes(4, 2 ** 30, 2 ** 30)
    assert ctx.ds_decode_shared_workspace_bytes(100000, 4000, 4000) >= ctx.ds_decode_shared_workspace_bytes(65535, 4000, 4000)
    ctx.close()


def test_more_than_a_launch_can_have():
    ctx = binding.Context(1024, 8, 128, 1024, n_kv_heads=2)
    w = binding.LayerWeights()
    for name, _ in binding.LayerWeights._fields_:
        setattr(w, name, P)
    w, end, cache = ctypes.byref(w), (P, 1 << 50, None), (*CACHE, 1)
    lib, h = ctx.lib, ctx.handle
    assert lib.ds_decode_attention_quant(h, P, P, P, 65536, 2, 32, *cache, P, *end) == INVALID
    assert lib.ds_decode_step_quant(h, w, P, P, P, 65536, 2, 32, *cache, 2 * P, *end) == INVALID
    for B, groups, rows in ((65536, 2, 40000), (40000, 40000, 40000), (8, 2 ** 31 - 1, 8)):
        assert lib.ds_decode_attention_shared(h, P, P, groups, rows, P, P, 400, 6400, P, P, B, 2, 32, *cache, P, *end) == INVALID
        assert lib.ds_decode_step_shared(h, w, P, P, groups, rows, P, P, 400, 6400, P, P, B, 2, 32, *cache, 2 * P, *end) == INVALID
    ctx.close()
