"""The 8-bit cache and shared prefixes as a serving loop uses them: prompts through ds_prefill, handed off quantised, decoded
step by step; and the debug validation of the calls' index arrays."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu
from tests.kv_pages import KINDS

pytestmark = pytest.mark.gpu

LAYERS = [synth.TINY, synth.ModelShape(hidden=1024, n_heads=8, head_dim=128, ffn=2048, n_kv_heads=2)]


def _pages(kind, nb, shape):
    """Poisoned pages of a kind: NaN wherever nothing is written."""
    n, s = shape.kv_heads, shape.head_dim
    if kind == binding.KV_BF16:
        k = torch.full((nb, n, 16, s), float("nan"), dtype=torch.bfloat16, device="cuda")
        return k, k.clone(), None, None
    k = torch.full((nb, n, 16, s), 0x7f, dtype=torch.uint8, device="cuda")
    sc = torch.full((nb, n, 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    return k, k.clone().view(nb, n, s, 16), sc, sc.clone()


def _tokens(pages, kind, table, length):
    """K and V of a sequence as its pages hold them, in 64 bits."""
    at = [int(p) for p in table[:-(-length // 16)]]
    k, v, ks, vs = pages
    if kind == binding.KV_BF16:
        return [gu.to_f64(x[at]).transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[:length] for x in (k, v)]
    k = kvo.stands_for(k[at].cpu().numpy(), gu.to_f64(ks[at]), kind)
    v = kvo.stands_for(v[at].cpu().numpy().transpose(0, 1, 3, 2), gu.to_f64(vs[at]), kind)
    return [x.transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[:length] for x in (k, v)]


def _check_step(w, shape, x, y, new_rows, keys, kind):
    """y of a step whose rows attend over keys[i] = (k, v), the new row the last of them, against the layer in 64 bits; and
    the new rows against the projection's.  Tolerances: those of the other layer tests (1e-2 of the largest, gpu_util's
    for the update); a new row is a bf16 product's (1e-2 of its largest), and rounded by half a step of its format: e4m3
    2^-4 of a number and 2^-10 of the scale where numbers are small, int8 half the scale."""
    a = orc.layernorm(x, w["ln1_g"], w["ln1_b"], shape.ln_eps)
    q, k, v = orc._split_qkv(orc.linear(a, w["w_qkv"], w["b_qkv"]), shape.n_heads, shape.head_dim)
    o = np.zeros((len(x), shape.n_heads, shape.head_dim))
    for i, (kk, vv) in enumerate(keys):
        if len(kk):
            o[i] = kvo.attend(q[i], kk, vv)[0]
        for got, want in ((kk, k), (vv, v)):
            if not new_rows[i]:
                continue
            most = np.abs(want[i]).max(-1, keepdims=True)
            half = {0: 2.0 ** -8 * np.abs(want[i]), 1: 2.0 ** -4 * np.abs(want[i]) + 2.0 ** -10 * most / 224,
                    2: most / 127 * 0.5 * (1 + 2.0 ** -7)}[kind]
            assert (np.abs(got[-1] - want[i]) <= half * 1.02 + 1e-2 * most).all()
    want = orc._post_attention(w, x, o, shape.ln_eps)
    got = gu.to_f64(y)
    assert gu.rel_err(got, want) <= 1e-2 and gu.update_ok(got, want, x)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("shape", LAYERS, ids=["tiny", "gqa"])
def test_a_request_on_pages_of_8_bits(gpu, shape, kind):
    kind, lens, steps, seed = KINDS[kind], [32, 19, 1], 4, 5
    ctx, h, B, t = gu.make_ctx(shape), shape.hidden, 3, 52
    wbits = synth.make_layer_weights(shape, seed)
    lw, _keep = gu.weights_to_dev(wbits)
    w = orc.weights_from_bits(wbits)
    x = gu.to_dev(synth.make_activations(t, h, seed))
    y = torch.empty_like(x)
    k_out, v_out = (torch.empty(t, shape.kv_heads, shape.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu = gu.i32_dev(synth.cu_seqlens(lens))
    ctx.ds_prefill(lw, x, cu, B, t, max(lens), y, k_out, v_out, gu.workspace(ctx.ds_prefill_workspace_bytes(t)))
    table, nb = synth.make_block_tables([l + steps for l in lens] + [16], 16, seed)
    table = table[:4]
    bt, pages = gu.i32_dev(table), _pages(kind, nb, shape)
    ctx.ds_kv_migrate_quant(k_out, v_out, cu, B, t, max(lens), bt, table.shape[1], *pages, nb, kind)
    # back as rows: what another pass over the prompt would start from, one rounding from what was handed off
    back = torch.empty((2,) + tuple(k_out.shape), dtype=torch.bfloat16, device="cuda")
    ctx.ds_kv_read_quant(cu, B, t, max(lens), bt, table.shape[1], *pages, nb, kind, back[0], back[1])
    torch.cuda.synchronize()
    for got, rows in zip(back, (k_out, v_out)):
        rows = gu.to_f64(rows)
        most = np.abs(rows).max(-1, keepdims=True)
        half = (2.0 ** -4 * np.abs(rows) + 2.0 ** -10 * most / 224 if kind == binding.KV_E4M3 else most / 127 * 0.51)
        assert (np.abs(gu.to_f64(got) - rows) <= half + 2.0 ** -8 * most).all()
    # a fourth row pads the batch
    ctx_lens = np.array(lens + [-1], np.int32)
    ws = gu.workspace(ctx.ds_decode_quant_workspace_bytes(4, max(lens) + steps))
    for step in range(steps):
        xn = synth.make_activations(4, h, seed, stream=1 + step)
        yd = torch.empty(4, h, dtype=torch.bfloat16, device="cuda")
        before = [p.clone() for p in pages]
        ctx.ds_decode_step_quant(lw, gu.to_dev(xn), gu.i32_dev(ctx_lens), bt, 4, table.shape[1], int(ctx_lens.max()) + 1,
                                 *pages, nb, kind, yd, ws)
        torch.cuda.synchronize()
        keys = [_tokens(pages, kind, table[i], int(l) + 1) for i, l in enumerate(ctx_lens)]
        _check_step(w, shape, orc.from_bf16_bits(xn), yd, [True] * 3 + [False], keys, kind)
        # nothing but the three new slots changed
        for a, b, slot_axis in zip(before, pages, (2, 3, 2, 2)):
            a, b = (z.view(torch.uint8) if z.dtype == torch.uint8 else z.view(torch.int16) for z in (a, b))
            same = (a == b).movedim(slot_axis, 1).flatten(2).all(2)
            for i in range(3):
                same[int(table[i][ctx_lens[i] // 16]), int(ctx_lens[i]) % 16] = True
            assert same.all()
        ctx_lens[:3] += 1


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("shape", LAYERS, ids=["tiny", "gqa"])
def test_continuations_of_shared_prompts(gpu, shape, kind):
    """Two prompts handed off once each; three and two continuations of them, from no token of their own on."""
    kind, prompts, rows_of, steps, seed = KINDS[kind], [45, 16], [3, 2], 18, 9
    ctx, h, B, t = gu.make_ctx(shape), shape.hidden, 5, 61
    wbits = synth.make_layer_weights(shape, seed)
    lw, _keep = gu.weights_to_dev(wbits)
    w = orc.weights_from_bits(wbits)
    x = gu.to_dev(synth.make_activations(t, h, seed))
    y = torch.empty_like(x)
    k_out, v_out = (torch.empty(t, shape.kv_heads, shape.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu = gu.i32_dev(synth.cu_seqlens(prompts))
    ctx.ds_prefill(lw, x, cu, 2, t, max(prompts), y, k_out, v_out, gu.workspace(ctx.ds_prefill_workspace_bytes(t)))
    table, nb = synth.make_block_tables(prompts + [steps] * B, 16, seed)
    pt, bt, pages = gu.i32_dev(table[:2]), gu.i32_dev(table[2:]), _pages(kind, nb, shape)
    if kind == binding.KV_BF16:
        ctx.ds_kv_migrate(k_out, v_out, cu, 2, t, max(prompts), pt, table.shape[1], pages[0], pages[1], nb)
    else:
        ctx.ds_kv_migrate_quant(k_out, v_out, cu, 2, t, max(prompts), pt, table.shape[1], *pages, nb, kind)
    cug = np.concatenate([[0], np.cumsum(rows_of)])
    ws = gu.workspace(ctx.ds_decode_shared_workspace_bytes(B, max(prompts), steps))
    lens = np.zeros(B, np.int32)
    for step in range(steps):
        xn = synth.make_activations(B, h, seed, stream=1 + step)
        yd = torch.empty(B, h, dtype=torch.bfloat16, device="cuda")
        ctx.ds_decode_step_shared(lw, gu.to_dev(xn), gu.i32_dev(cug), 2, 3, gu.i32_dev(prompts), pt, table.shape[1],
                                  max(prompts), gu.i32_dev(lens), bt, B, table.shape[1], step + 1, *pages, nb, kind, yd, ws)
        torch.cuda.synchronize()
        lens += 1
        if step not in (0, 1, 15, 16, 17):
            continue
        keys = []
        for i in range(B):
            g = int(np.searchsorted(cug, i, side="right") - 1)
            (kp, vp), (kk, vv) = _tokens(pages, kind, table[g], prompts[g]), _tokens(pages, kind, table[2 + i], step + 1)
            keys.append((np.concatenate([kp, kk]), np.concatenate([vp, vv])))
        _check_step(w, shape, orc.from_bf16_bits(xn), yd, [True] * B, keys, kind)


def test_a_step_replays_from_a_graph(gpu):
    """Both steps captured, three replays with other inputs and one token more each, eager work between them."""
    shape = synth.ModelShape(hidden=1024, n_heads=8, head_dim=128, ffn=2048)
    ctx, h, B, seed, kind = gu.make_ctx(shape), shape.hidden, 6, 3, binding.KV_E4M3
    lw, _keep = gu.weights_to_dev(synth.make_layer_weights(shape, seed))
    table, nb = synth.make_block_tables([700, 40] + [60] * B, 16, seed)
    pt, bt, mb = gu.i32_dev(table[:2]), gu.i32_dev(table[2:]), table.shape[1]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    k = torch.randn(nb, shape.kv_heads, 16, 128, device="cuda", generator=gen) * 30
    pages = [k.to(torch.float8_e4m3fn).view(torch.uint8), (k + 1).to(torch.float8_e4m3fn).view(torch.uint8).view(nb, -1, 128, 16),
             torch.full((nb, shape.kv_heads, 16), 2.0 ** -5, dtype=torch.bfloat16, device="cuda"),
             torch.full((nb, shape.kv_heads, 16), 2.0 ** -5, dtype=torch.bfloat16, device="cuda")]
    cug, pl = gu.i32_dev([0, 4, 6]), gu.i32_dev([700, 40])
    lens = gu.i32_dev([0, 3, 40, 15, 16, 50])
    x = torch.randn(B, h, device="cuda", generator=gen).bfloat16()
    ws = gu.workspace(max(ctx.ds_decode_shared_workspace_bytes(B, 700, 60), ctx.ds_decode_quant_workspace_bytes(B, 60)))

    def steps(p, y1, y2):
        ctx.ds_decode_step_quant(lw, x, lens, bt, B, mb, 60, *p, nb, kind, y1, ws)
        ctx.ds_decode_step_shared(lw, x, cug, 2, 4, pl, pt, mb, 700, lens, bt, B, mb, 60, *p, nb, kind, y2, ws)

    y1, y2, e1, e2 = (torch.empty_like(x) for _ in range(4))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        steps([p.clone() for p in pages], e1, e2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        steps(pages, y1, y2)
    for i in range(3):
        x.copy_(torch.randn(B, h, device="cuda", generator=gen).bfloat16())
        eager = [p.clone() for p in pages]
        graph.replay()
        torch.cuda.synchronize()
        steps(eager, e1, e2)
        torch.cuda.synchronize()
        assert torch.equal(y1, e1) and torch.equal(y2, e2), i
        assert torch.isfinite(y1.float()).all() and torch.isfinite(y2.float()).all()
        for a, b in zip(pages, eager):
            assert torch.equal(a, b), i
        lens += 1


def _bounds(call, text):
    with pytest.raises(binding.DsError) as e:
        call()
    assert e.value.status == 5 and text in str(e.value), str(e.value)


def test_validation_of_index_arrays(gpu):
    """Copied back and refused before anything is launched."""
    shape = synth.TINY
    ctx, h = gu.make_ctx(shape), shape.hidden
    ctx.ds_set_validate(True)
    lw, _keep = gu.weights_to_dev(synth.make_layer_weights(shape, 1))
    nb, kind = 8, binding.KV_INT8
    pages = _pages(kind, nb, shape)
    rows = torch.zeros(40, 4, 64, dtype=torch.bfloat16, device="cuda")
    x, y, q = (torch.zeros(2, h, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    good = gu.i32_dev([[0, 1], [2, 3]])
    ws = gu.workspace(ctx.ds_decode_shared_workspace_bytes(2, 32, 32))
    cache = (*pages, nb, kind)
    cu = gu.i32_dev([0, 20, 40])

    def migrate(cu, bt):
        ctx.ds_kv_migrate_quant(rows, rows, cu, 2, 40, 20, bt, 2, *cache)
        ctx.ds_kv_read_quant(cu, 2, 40, 20, bt, 2, *cache, rows, rows.clone())

    migrate(cu, good)
    for bad_cu, text in (([1, 20, 40], "cu_seqlens[0]"), ([0, 20, 39], "must be t"), ([0, 21, 40], "max_seqlen")):
        _bounds(lambda: migrate(gu.i32_dev(bad_cu), good), text)
        _bounds(lambda: ctx.ds_kv_read_quant(gu.i32_dev(bad_cu), 2, 40, 20, good, 2, *cache, rows, rows), text)
    for bad in ([[0, 8], [2, 3]], [[0, 1], [2, -1]]):
        _bounds(lambda: migrate(cu, gu.i32_dev(bad)), "block_tables")
        _bounds(lambda: ctx.ds_kv_read_quant(cu, 2, 40, 20, gu.i32_dev(bad), 2, *cache, rows, rows), "block_tables")

    def append(lens, bt=good):
        ctx.ds_kv_append_quant(rows, rows, 256, gu.i32_dev(lens), bt, 2, 2, *cache)

    append([31, -1])
    _bounds(lambda: append([32, 0]), "outside [0, 32]")
    _bounds(lambda: append([0, -2]), "outside [0, 32]")
    _bounds(lambda: append([16, 0], gu.i32_dev([[0, -1], [1, 2]])), "block_tables[0][1]")

    def attend(lens, bt=good):
        ctx.ds_decode_attention_quant(q, gu.i32_dev(lens), bt, 2, 2, 32, *cache, y, ws)

    attend([0, 32])
    _bounds(lambda: attend([0, 33]), "sequence 1")
    _bounds(lambda: attend([1, 17], gu.i32_dev([[0, 1], [2, 8]])), "block_tables[1][1]")

    def step(lens, bt=good):
        ctx.ds_decode_step_quant(lw, x, gu.i32_dev(lens), bt, 2, 2, 32, *cache, y, ws)

    step([-1, 31])
    _bounds(lambda: step([0, 32]), "sequence 1")
    _bounds(lambda: step([16, 0], gu.i32_dev([[0, -1], [2, 3]])), "block_tables[0][1]")

    def shared(cug=(0, 1, 2), prefix=(32, 0), pt=((4, 5), (-1, -1)), lens=(0, 32), whole=False):
        g = (gu.i32_dev(cug), 2, 2, gu.i32_dev(prefix), gu.i32_dev(pt), 2, 32)
        if whole:
            ctx.ds_decode_step_shared(lw, x, *g, gu.i32_dev(np.array(lens) - 1), good, 2, 2, 32, *cache, y, ws)
        else:
            ctx.ds_decode_attention_shared(q, *g, gu.i32_dev(lens), good, 2, 2, 32, *cache, y, ws)

    for whole in (False, True):
        shared(whole=whole)
        for bad, text in ((dict(cug=(0, 1, 1)), "cu_groups"), (dict(cug=(1, 1, 2)), "cu_groups"),
                          (dict(cug=(0, 3, 2)), "group 0"), (dict(prefix=(33, 0)), "prefix 0"),
                          (dict(prefix=(0, -1)), "prefix 1"), (dict(prefix=(32, 1)), "block_tables[1][0]"),
                          (dict(pt=((4, 8), (-1, -1))), "block_tables[0][1]"), (dict(lens=(33, 1)), "sequence 0")):
            _bounds(lambda: shared(whole=whole, **bad), text)
    torch.cuda.synchronize()
