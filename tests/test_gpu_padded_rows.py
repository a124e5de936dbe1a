"""Rows of ctx_lens = -1 in ds_decode_step_shared: one meaning on every kind of pages.  Nothing is written for them, whichever
of the kernels it is that appends on bf16 pages, and they attend over their group's prefix alone."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu
from tests.kv_pages import Cache

pytestmark = pytest.mark.gpu


def _layer(heads, head_dim, n_kv, ffn=512):
    return synth.ModelShape(hidden=heads * head_dim, n_heads=heads, head_dim=head_dim, ffn=ffn, n_kv_heads=n_kv)


def _bits(cache):
    return [p.view(torch.uint8 if p.dtype == torch.uint8 else torch.int16).clone()
            for p in (cache.k, cache.v, cache.ks, cache.vs) if p is not None]


def _step(ctx, lw, c, x, cug, prefix, own, tables):
    """One step on the pages of `c`, whose first sequences are the prefixes; returns y."""
    B, (pt, bt) = len(own), tables
    y, groups = torch.full_like(x, 9.0), len(prefix)
    ws = gu.workspace(ctx.ds_decode_shared_workspace_bytes(B, max(prefix), 40))
    ctx.ds_decode_step_shared(lw, x, gu.i32_dev(cug), groups, int(np.diff(cug).max()), gu.i32_dev(prefix), gu.i32_dev(pt),
                              pt.shape[1], max(prefix), gu.i32_dev(own), gu.i32_dev(bt), B, bt.shape[1], 40, *c.args, y, ws)
    torch.cuda.synchronize()
    return y


def _case(shape, kind, B, seed):
    """Two groups; of their rows every third pads.  Pages poisoned wherever no token is, -1 where a row needs none."""
    prefix, cug = [45, 16], [0, B // 2, B]
    own = [-1 if i % 3 == 0 else (7 * i) % (33 if B < 1000 else 3) for i in range(B)]
    lens = prefix + [max(l, 0) for l in own]
    c = Cache(kind, lens, shape.kv_heads, shape.head_dim, seed, room=prefix + [l + 1 for l in lens[2:]])
    table = np.array(c.table)
    bt = table[2:].copy()
    spare = [int(bt[i, 0]) for i in range(B) if own[i] < 0]
    for i in range(B):
        if own[i] < 0:
            bt[i] = -1
    return prefix, cug, own, c, table[:2], bt, spare


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("heads,head_dim,n_kv,B,plan", [
    (4, 64, 0, 6, (True, False)),        # written by the unsplit product itself
    (16, 128, 0, 12, (True, False)),
    (40, 128, 0, 40, (True, False)),
    (20, 128, 4, 40, (True, True)),      # by the pass that adds up its splits
    (20, 128, 4, 100, (False, True)),
    (8, 128, 2, 100, (False, False)),    # by the tile kernel's epilogue
    (4, 64, 0, 6000, (False, False)),    # by a launch of its own (a tile that does not write pages)
])
def test_nothing_is_written_for_a_row_that_pads(gpu, heads, head_dim, n_kv, B, plan, kind):
    shape = _layer(heads, head_dim, n_kv)
    ctx = gu.make_ctx(shape)
    p = ctx.ds_layer_plan(B, shape.hidden, shape.qkv_width)
    assert (p["streaming"], p["splits"] > 1) == plan
    lw, _keep = gu.dev_layer_weights(shape, 3)
    prefix, cug, own, c, pt, bt, spare = _case(shape, kind, B, 11)
    x = gu.dev_normal_bits((B, shape.hidden), 1.0, 4)
    before = _bits(c)
    y = _step(ctx, lw, c, x, cug, prefix, own, (pt, bt))
    live = [i for i in range(B) if own[i] >= 0]
    page = torch.tensor([int(bt[i, own[i] // 16]) for i in live], device="cuda")
    slot = torch.tensor([own[i] % 16 for i in live], device="cuda")
    for a, b, axis in zip(before, _bits(c), (2, 2, 2, 2) if kind == "bf16" else (2, 3, 2, 2)):
        changed = (a != b).movedim(axis, 1).flatten(2).any(2)        # [pages, slots]
        want = torch.zeros_like(changed)
        want[page, slot] = True
        assert not (changed & ~want).any(), torch.nonzero(changed & ~want)[:4]
        assert changed[page, slot].all()
    # the other rows: the bits that they have beside rows with a token of their own
    full = [max(l, 0) for l in own]
    table = bt.copy()
    for i, blk in zip([i for i in range(B) if own[i] < 0], spare):
        table[i, 0] = blk
    c2 = Cache(kind, c.lens, shape.kv_heads, shape.head_dim, 11, room=prefix + [l + 1 for l in c.lens[2:]])
    y2 = _step(ctx, lw, c2, x, cug, prefix, full, (pt, table))
    assert torch.equal(y[live], y2[live])
    assert torch.isfinite(y.float()).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("shape", [synth.TINY, _layer(8, 128, 2, 1024)], ids=["tiny", "gqa"])
def test_a_row_that_pads_attends_over_its_prefix(gpu, shape, kind):
    """Against the layer in 64 bits; tolerances of the other layer tests."""
    ctx, B = gu.make_ctx(shape), 7
    wbits = synth.make_layer_weights(shape, 5)
    lw, _keep = gu.weights_to_dev(wbits)
    w = orc.weights_from_bits(wbits)
    prefix, cug, own, c, pt, bt, _ = _case(shape, kind, B, 21)
    xbits = synth.make_activations(B, shape.hidden, 6)
    y = _step(ctx, lw, c, gu.to_dev(xbits), cug, prefix, own, (pt, bt))
    x = orc.from_bf16_bits(xbits)
    a = orc.layernorm(x, w["ln1_g"], w["ln1_b"], shape.ln_eps)
    q, _k, _v = orc._split_qkv(orc.linear(a, w["w_qkv"], w["b_qkv"]), shape.n_heads, shape.head_dim)
    pads = [i for i in range(B) if own[i] < 0]
    o = np.stack([kvo.attend(q[i], *c.seq(0 if i < cug[1] else 1))[0] for i in pads])
    want, got = orc._post_attention(w, x[pads], o, shape.ln_eps), gu.to_f64(y)[pads]
    assert gu.rel_err(got, want) <= 1e-2 and gu.update_ok(got, want, x[pads])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_debug_validation_takes_it(gpu, kind):
    shape = synth.TINY
    ctx = gu.make_ctx(shape)
    ctx.ds_set_validate(True)
    lw, _keep = gu.weights_to_dev(synth.make_layer_weights(shape, 1))
    prefix, cug, own, c, pt, bt, _ = _case(shape, kind, 5, 2)
    x = gu.dev_normal_bits((5, shape.hidden), 1.0, 4)
    _step(ctx, lw, c, x, cug, prefix, own, (pt, bt))
    with pytest.raises(binding.DsError) as e:
        _step(ctx, lw, c, x, cug, prefix, [-2] + own[1:], (pt, bt))
    assert e.value.status == 5 and "sequence 0" in str(e.value)
