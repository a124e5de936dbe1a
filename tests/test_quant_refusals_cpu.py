"""What the calls for the 8-bit cache and for shared prefixes refuse before anything touches a device, and what their
workspace queries promise."""
import ctypes

import pytest

from paper_2401_09670_amd import binding

P = 4096            # an aligned address that nobody follows: every call here is refused on the host
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(1024, 8, 128, 1024, n_kv_heads=2)
    yield c
    c.close()


def _weights():
    w = binding.LayerWeights()
    for name, _ in binding.LayerWeights._fields_:
        setattr(w, name, P)
    return w


CACHE = dict(k_cache=P, v_cache=P, k_scale=P, v_scale=P, num_blocks=64, kv_type=1)
GROUPS = dict(cu_groups=P, n_groups=2, max_group_rows=3, prefix_lens=P, prefix_tables=P, max_prefix_blocks=4,
              max_prefix_len=64)
ROWS = dict(cu_seqlens=P, B=2, t=40, max_seqlen=30, block_tables=P, max_blocks=2)
END = dict(workspace=P, workspace_bytes=1 << 30)
CALLS = {  # arguments in their order, without the context and the stream
    "ds_kv_migrate_quant": dict(k_src=P, v_src=P, **ROWS, **CACHE),
    "ds_kv_read_quant": dict(**ROWS, **CACHE, k_dst=P, v_dst=P),
    "ds_kv_append_quant": dict(k_new=P, v_new=P, row_stride=256, ctx_lens=P, block_tables=P, B=4, max_blocks=2, **CACHE),
    "ds_decode_attention_quant": dict(q=P, kv_lens=P, block_tables=P, B=4, max_blocks=128, max_kv_len=2000, **CACHE, o=P, **END),
    "ds_decode_attention_shared": dict(q=P, **GROUPS, kv_lens=P, block_tables=P, B=4, max_blocks=2, max_kv_len=32, **CACHE,
                                       o=P, **END),
    "ds_decode_step_quant": dict(weights=None, x=P, ctx_lens=P, block_tables=P, B=4, max_blocks=2, max_ctx=32, **CACHE, y=2 * P,
                                 **END),
    "ds_decode_step_shared": dict(weights=None, x=P, **GROUPS, ctx_lens=P, block_tables=P, B=4, max_blocks=2, max_ctx=32,
                                  **CACHE, y=2 * P, **END),
}


def _status(ctx, name, **change):
    args = dict(CALLS[name])
    assert set(change) <= set(args), change
    args.update(change)
    if "weights" in args and "weights" not in change:
        args["weights"] = ctypes.byref(_weights())
    return getattr(ctx.lib, name)(ctx.handle, *args.values(), None)


def _cases():
    for name, args in CALLS.items():
        for a, v in args.items():
            if a in ("workspace", "workspace_bytes", "weights"):
                continue
            if v in (P, 2 * P):
                yield name, {a: None}, INVALID
                if a not in ("cu_seqlens", "block_tables", "ctx_lens", "kv_lens", "cu_groups", "prefix_lens", "prefix_tables"):
                    yield name, {a: P + 8}, INVALID            # not 16-byte aligned
            elif a != "kv_type":
                yield name, {a: 0}, INVALID
                yield name, {a: -1}, INVALID
        for kind in (3, -1) + (() if "shared" in name else (0,)):
            yield name, dict(kv_type=kind), UNSUPPORTED
        if "shared" in name:
            yield name, dict(kv_type=0), INVALID               # bf16 pages come without scales
            yield name, dict(max_group_rows=1), INVALID        # 2 groups of 1 cannot hold 4 rows
            yield name, dict(max_prefix_len=65), INVALID       # beyond the table
        if "max_seqlen" in args:
            yield name, dict(max_seqlen=33), INVALID
            yield name, dict(max_seqlen=41, max_blocks=9), INVALID
        if "max_kv_len" in args:
            yield name, dict(max_kv_len=16 * args["max_blocks"] + 1), INVALID
        if "max_ctx" in args:
            yield name, dict(max_ctx=33), INVALID
            yield name, dict(y=P), INVALID                     # in place of x
            yield name, dict(weights=None), INVALID
            yield name, dict(weights=ctypes.byref(binding.LayerWeights())), INVALID
        if "workspace" in args:
            yield name, dict(workspace=None), WORKSPACE
            yield name, dict(workspace_bytes=64), WORKSPACE
            yield name, dict(workspace=P + 8), INVALID
        if "row_stride" in args:
            yield name, dict(row_stride=248), INVALID          # below n_kv s
            yield name, dict(row_stride=260), INVALID          # rows that would not be aligned


@pytest.mark.parametrize("name,change,want", list(_cases()), ids=lambda v: str(v) if not isinstance(v, dict) else
                         ",".join(f"{a}" for a in v))
def test_refused(ctx, name, change, want):
    assert _status(ctx, name, **change) == want
    text = binding.load_library().ds_last_error(ctx.handle).decode()
    assert name in text or "weight" in text, text


@pytest.mark.parametrize("name", list(CALLS))
def test_no_context(name):
    args = dict(CALLS[name])
    if "weights" in args:
        args["weights"] = ctypes.byref(_weights())
    assert getattr(binding.load_library(), name)(None, *args.values(), None) == INVALID


@pytest.mark.parametrize("hidden,n,s,ffn,n_kv", [(256, 4, 64, 1024, 0), (5120, 40, 128, 20480, 0), (8192, 64, 128, 28672, 8),
                                                 (2048, 16, 128, 4096, 1)])
def test_a_workspace_for_a_maximum_serves_smaller_calls(hidden, n, s, ffn, n_kv):
    ctx = binding.Context(hidden, n, s, ffn, n_kv_heads=n_kv)
    for B, L, X in ((1, 16, 16), (7, 300, 5000), (64, 4096, 700), (256, 2048, 2048)):
        quant, shared = ctx.ds_decode_quant_workspace_bytes(B, L), ctx.ds_decode_shared_workspace_bytes(B, X, L)
        assert 0 < quant <= shared
        for b in {1, 2, B // 2 or 1, B}:
            for l in (1, L // 3 or 1, L):
                assert ctx.ds_decode_quant_workspace_bytes(min(b, B), l) <= quant
                for x in (1, X // 2, X):
                    assert ctx.ds_decode_shared_workspace_bytes(min(b, B), x, l) <= shared


def test_sizes_of_nothing():
    ctx = binding.Context(256, 4, 64, 1024)
    assert ctx.ds_decode_quant_workspace_bytes(0, 5) == 0 and ctx.ds_decode_quant_workspace_bytes(5, 0) == 0
    assert ctx.ds_decode_shared_workspace_bytes(5, 0, 5) == 0 and ctx.ds_decode_shared_workspace_bytes(0, 5, 5) == 0
    assert binding.load_library().ds_decode_quant_workspace_bytes(None, 1, 1) == 0
