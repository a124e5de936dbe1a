"""What the calls for positions by rotation and for attention through a window refuse before anything touches a device."""
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
