"""What the calls for positions by rotation and for attention through a window refuse before anything touches a device."""
import random
import re

import pytest

from paper_2401_09670_amd import binding

P = 4096            # an aligned address that nobody follows: every call here is refused on the host
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(1024, 8, 128, 1024, n_kv_heads=2)
    yield c
    c.close()


CACHE = dict(k_cache=P, v_cache=P, k_scale=P, v_scale=P, num_blocks=64, kv_type=1)
CALLS = {  # arguments in their order, without the context and the stream
    "ds_kv_append_rotary": dict(q=P, q_stride=1536, k=P, v=P, kv_stride=1536, cu_rows=P, B=2, t=40, ctx_lens=P, positions=P,
                                table=P, n_pos=100, rot=64, adjacent=0, block_tables=P, max_blocks=4, **CACHE, q_out=2 * P,
                                k_out=2 * P),
    "ds_prefill_attention_window": dict(q=P, q_stride=1536, k=P, k_stride=256, v=P, v_stride=1536, cu_seqlens=P, B=2, t=40,
                                        max_seqlen=30, window=8, sinks=4, o=P),
    "ds_decode_attention_window": dict(q=P, kv_lens=P, block_tables=P, B=4, max_blocks=128, max_kv_len=2000, window=1900,
                                       sinks=4, **CACHE, o=P, workspace=P, workspace_bytes=1 << 30),
}
MAY_BE_NULL = ("cu_rows", "positions", "k_out")
INDICES = ("cu_rows", "cu_seqlens", "ctx_lens", "positions", "block_tables", "kv_lens")


def _status(ctx, name, **change):
    args = dict(CALLS[name])
    assert set(change) <= set(args), change
    args.update(change)
    return getattr(ctx.lib, name)(ctx.handle, *args.values(), None)


def _cases():
    for name, args in CALLS.items():
        for a, v in args.items():
            if a in ("workspace", "workspace_bytes", "kv_type", "adjacent", "sinks"):
                continue
            if v in (P, 2 * P):
                if a not in MAY_BE_NULL:
                    yield name, {a: None}, INVALID
                if a not in INDICES:
                    yield name, {a: P + 8}, INVALID            # not 16-byte aligned
            else:
                bad = UNSUPPORTED if a == "rot" else INVALID
                yield name, {a: 0}, bad
                yield name, {a: -1}, bad
        if "kv_type" in args:
            for kind in (3, -1):
                yield name, dict(kv_type=kind), UNSUPPORTED
            yield name, dict(kv_type=0), INVALID               # bf16 pages come without scales
            yield name, dict(kv_type=0, k_scale=None), INVALID
        for a in ("q_stride", "k_stride", "v_stride") if "max_seqlen" in args else ():
            for stride in (248, args[a] + 4, 2 ** 24 + 8):     # below a row's width, not aligned, too far apart
                yield name, {a: stride}, INVALID
        if "max_seqlen" in args:
            yield name, dict(max_seqlen=41), INVALID
            yield name, dict(B=2 ** 31 - 1), INVALID           # more than a launch can have
        if "window" in args:
            yield name, dict(window=-2 ** 31), INVALID
            yield name, dict(sinks=-1), INVALID
        if "workspace" in args:
            yield name, dict(workspace=None), WORKSPACE
            yield name, dict(workspace_bytes=64), WORKSPACE
            yield name, dict(workspace=P + 8), INVALID
            yield name, dict(max_kv_len=16 * args["max_blocks"] + 1), INVALID
            yield name, dict(B=65536), INVALID                 # more than a launch can have
            yield name, dict(max_kv_len=2 ** 31 - 1, max_blocks=2 ** 27), INVALID
    name = "ds_kv_append_rotary"
    for stride in (dict(q_stride=1016), dict(kv_stride=248), dict(q_stride=1028), dict(kv_stride=260)):
        yield name, stride, INVALID                            # below a row's width, rows that would not be aligned
    for rot in (8, 24, 40, 144, 256):
        yield name, dict(rot=rot), UNSUPPORTED
    yield name, dict(cu_rows=None), INVALID                    # 40 rows of 2 sequences, one each
    yield name, dict(q_out=P), INVALID                         # in place, rows apart
    yield name, dict(k_out=P), INVALID
    yield name, dict(t=2 ** 31 - 1), INVALID                   # more than a launch can have


@pytest.mark.parametrize("name,change,want", list(_cases()), ids=lambda v: str(v) if not isinstance(v, dict) else
                         ",".join(f"{a}={b}" for a, b in v.items()))
def test_refused(ctx, name, change, want):
    assert _status(ctx, name, **change) == want
    text = binding.load_library().ds_last_error(ctx.handle).decode()
    assert name in text, text


@pytest.mark.parametrize("name", list(CALLS))
def test_no_context(name):
    assert getattr(binding.load_library(), name)(None, *CALLS[name].values(), None) == INVALID


SHAPES = [(256, 4, 64, 0), (5120, 40, 128, 0), (8192, 64, 128, 8), (2048, 16, 128, 1), (4096, 32, 128, 1)]


@pytest.mark.parametrize("hidden,n,s,n_kv", SHAPES)
def test_a_decode_call_needs_no_more_than_was_promised(hidden, n, s, n_kv):
    """A workspace for the largest batch, length, window and first tokens serves every smaller call."""
    c = binding.Context(hidden, n, s, 1024, n_kv_heads=n_kv)
    rng, asked = random.Random(hidden), 0
    for _ in range(1500):
        B, L = int(2 ** rng.uniform(0, 8.5)), int(2 ** rng.uniform(0, 16))
        window, sinks = int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 10)) - 1
        most = [x + rng.randrange(x + 1) for x in (B, L, window, sinks)]
        kind = rng.randrange(3)
        scales = (None, None) if kind == 0 else (P, P)
        promised = c.ds_decode_window_workspace_bytes(*most)
        st = c.lib.ds_decode_attention_window(c.handle, P, P, P, B, -(-L // 16), L, window, sinks, P, P, *scales, 1 << 20, kind,
                                              P, None, 0, None) if _splits(c, B, L, window, sinks) else None
        if st is not None:
            assert st == WORKSPACE
            asked += 1
            text = c.lib.ds_last_error(c.handle).decode()
            assert int(re.search(r"workspace 0 < (\d+)", text).group(1)) <= promised
    assert asked >= 5
    c.close()


def _splits(c, B, L, window, sinks):
    """Whether such a call surely asks for a workspace (else it would be launched): 96 pages or more, few rows."""
    seen = min(-(-L // 16), window // 16)
    return seen >= 96 and B * (c.cfg.n_kv_heads or c.cfg.n_heads) <= 128


def test_sizes_of_nothing():
    c = binding.Context(256, 4, 64, 1024)
    for args in ((0, 5, 5, 5), (5, 0, 5, 5), (5, 5, 0, 5), (5, 5, 5, -1), (5, 2 ** 31 - 1, 5, 5)):
        assert c.ds_decode_window_workspace_bytes(*args) == 0
    assert c.ds_decode_window_workspace_bytes(4, 2 ** 30, 2 ** 31 - 1, 2 ** 31 - 1) > 0
    assert binding.load_library().ds_decode_window_workspace_bytes(None, 1, 1, 1, 1) == 0
    c.close()
