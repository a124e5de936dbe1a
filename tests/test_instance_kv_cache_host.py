"""Sizes and counts of a pool of 8 bits (host logic)."""
import pytest

from paper_2401_09670_amd import instance as inst
from paper_2401_09670_amd import synth


@pytest.mark.parametrize("shape", [synth.TINY, synth.OPT_66B, synth.ModelShape(8192, 64, 128, 32768, n_kv_heads=8)])
def test_bytes_of_a_token(shape):
    numbers = 2 * shape.kv_heads * shape.head_dim
    assert inst.kv_token_bytes(shape) == inst.kv_token_bytes(shape, "bf16") == 2 * numbers
    for kind in ("e4m3", "int8"):
        assert inst.kv_token_bytes(shape, kind) == numbers + 2 * 2 * shape.kv_heads


def test_the_same_memory_holds_about_twice_the_pages():
    cfg = synth.config(3)
    reqs = inst.requests_for(cfg, 48)
    a, b = inst.plan_for(cfg, reqs, 80.0), inst.plan_for(cfg, reqs, 80.0, "e4m3")
    assert a["page_bytes"] == 2 * 2 * 9216 * 16 * 64
    assert 1.9 < b["pool_blocks"] / a["pool_blocks"] < 2.0
    assert a["pool_blocks"] * a["page_bytes"] <= 80e9 and b["pool_blocks"] * b["page_bytes"] <= 80e9


def test_a_step_reads_fewer_bytes():
    shape, ctx = synth.OPT_13B, [500] * 64
    full, weights = inst.decode_bytes(ctx, shape, 1, 0), inst.decode_bytes([], shape, 1, 0)
    less = inst.decode_bytes(ctx, shape, 1, 0, "int8")
    assert (full - less) == 64 * 501 * (inst.kv_token_bytes(shape) - inst.kv_token_bytes(shape, "int8"))
    assert weights < less < full
