"""The three calls as a layer with rotated positions and a sliding window uses them: prompts appended and attended over, tokens
decoded one by one, pages behind the window given back; against 64 bits on what the calls before left."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from oracle import rotary_window_oracle as rwo
from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu
from tests.kv_pages import KINDS, close, rows
from tests.test_gpu_prefill_window import attend

pytestmark = pytest.mark.gpu


def _pages(kind, nb, n_kv, s):
    """NaN wherever nothing is written."""
    if kind == binding.KV_BF16:
        k = torch.full((nb, n_kv, 16, s), float("nan"), dtype=torch.bfloat16, device="cuda")
        return k, k.clone(), None, None
    k = torch.full((nb, n_kv, 16, s), 0x7f, dtype=torch.uint8, device="cuda")
    sc = torch.full((nb, n_kv, 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    return k, k.clone().view(nb, n_kv, s, 16), sc, sc.clone()


def _stands(bits, kind):
    """What a cache holds of bf16 rows."""
    x = orc.from_bf16_bits(bits)
    return x if kind == binding.KV_BF16 else kvo.stands_for(*kvo.quantise(x, kind), kind)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s,adjacent", [(8, 2, 64, False), (4, 4, 128, True), (16, 1, 64, False)])
def test_a_request(gpu, n, n_kv, s, adjacent, kind):
    kind, lens, window, sinks, steps, rot = KINDS[kind], [50, 3, 97], 33, 5, 20, s // 2 if adjacent else s
    ctx = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)
    rng, B, t, stride = np.random.default_rng(3), 3, sum(lens), (n + 2 * n_kv) * s
    table = rwo.angle_table(200, rot)
    table_dev = torch.from_numpy(table).cuda()
    bt, nb = synth.make_block_tables([l + steps for l in lens] + [16], 16, 7)       # a fourth row pads the batch
    pages = _pages(kind, nb, n_kv, s)

    def product(count):  # the rows of a QKV product, as bits
        return [rows(rng, count, h, s) for h in (n, n_kv, n_kv)]

    def turned(bits, at):
        return rwo.turned_bits(bits, table[at], adjacent)

    # the prompts
    q, k, v = product(t)
    flat = gu.to_dev(np.concatenate([q, k, v], 1).reshape(-1))
    cu = gu.i32_dev(synth.cu_seqlens(lens))
    q_out, k_out = (torch.empty(t, h, s, dtype=torch.bfloat16, device="cuda") for h in (n, n_kv))
    o = torch.empty_like(q_out)
    ctx.ds_kv_append_rotary(flat, stride, flat[n * s:], flat[(n + n_kv) * s:], stride, cu, B, t, gu.i32_dev([0] * 3), None,
                            table_dev, 200, rot, adjacent, gu.i32_dev(bt[:3]), bt.shape[1], *pages, nb, kind, q_out, k_out)
    ctx.ds_prefill_attention_window(q_out, n * s, k_out, n_kv * s, flat[(n + n_kv) * s:], stride, cu, B, t, max(lens), window,
                                    sinks, o)
    torch.cuda.synchronize()
    at = np.concatenate([np.arange(l) for l in lens])
    qt, kt = turned(q, at), turned(k, at)
    np.testing.assert_array_equal(gu.to_bits(q_out), qt)
    np.testing.assert_array_equal(gu.to_bits(k_out), kt)
    held, a = [], 0
    for l in lens:
        want, bound = attend(*(orc.from_bf16_bits(x[a:a + l]) for x in (qt, kt, v)), window, sinks)
        assert (np.abs(gu.to_f64(o)[a:a + l] - want) <= bound).all()
        held.append([kt[a:a + l], v[a:a + l]])
        a += l
    # tokens one by one; pages that the window has left behind are given back, and taken by others
    before, ws = np.array(lens + [-1]), gu.workspace(ctx.ds_decode_window_workspace_bytes(4, max(lens) + steps, window, sinks))
    qo, od = torch.empty(4, n, s, dtype=torch.bfloat16, device="cuda"), torch.empty(4, n, s, dtype=torch.bfloat16, device="cuda")
    for step in range(steps):
        q, k, v = product(4)
        flat = gu.to_dev(np.concatenate([q, k, v], 1).reshape(-1))
        ctx.ds_kv_append_rotary(flat, stride, flat[n * s:], flat[(n + n_kv) * s:], stride, None, 4, 4, gu.i32_dev(before), None,
                                table_dev, 200, rot, adjacent, gu.i32_dev(bt), bt.shape[1], *pages, nb, kind, qo)
        for i, l in enumerate(before[:3]):
            for p in range(-(-sinks // 16), (l + 1 - window) // 16):
                if bt[i, p] >= 0:
                    for x in pages:
                        if x is not None:
                            x[int(bt[i, p])] = float("nan") if x.dtype == torch.bfloat16 else 0x7f
                    bt[i, p] = -1
        ctx.ds_decode_attention_window(qo, gu.i32_dev(before + 1), gu.i32_dev(bt), 4, bt.shape[1], int(before.max()) + 1, window,
                                       sinks, *pages, nb, kind, od, ws)
        torch.cuda.synchronize()
        qt, kt = turned(q, np.maximum(before, 0)), turned(k, np.maximum(before, 0))
        np.testing.assert_array_equal(gu.to_bits(qo)[:3], qt[:3])
        for i in range(3):
            held[i] = [np.concatenate([x, y[i:i + 1]]) for x, y in zip(held[i], (kt, v))]
            kk, vv = (_stands(x, kind) for x in held[i])
            want, pav, size, keys = rwo.attend_window(orc.from_bf16_bits(qt[i]), kk, vv, window, sinks)
            assert not close(gu.to_f64(od[i]), want, pav, size, s, keys), (step, i)
        assert (od[3] == 0).all()
        before[:3] += 1
    assert (bt[2] < 0).any()


def test_a_piece_behind_its_beginning(gpu):
    """A prompt in two pieces leaves the cache that it leaves in one, and the second piece's queries, a sequence each over the
    pages of one table, see what they see in the whole prompt."""
    n, n_kv, s, l, cut, window, sinks = 8, 2, 64, 70, 41, 30, 4
    ctx = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)
    rng, stride = np.random.default_rng(4), (n + 2 * n_kv) * s
    bits = [rows(rng, l, h, s) for h in (n, n_kv, n_kv)]
    flat = gu.to_dev(np.concatenate(bits, 1).reshape(-1))
    table = torch.from_numpy(rwo.angle_table(100, s)).cuda()
    bt, nb = synth.make_block_tables([l], 16, 7)
    bt_dev, kind = gu.i32_dev(bt), binding.KV_E4M3
    whole, parts = _pages(kind, nb, n_kv, s), _pages(kind, nb, n_kv, s)
    q_out = torch.empty(l, n, s, dtype=torch.bfloat16, device="cuda")

    def append(pages, a, b):
        part = flat[a * stride:]
        ctx.ds_kv_append_rotary(part, stride, part[n * s:], part[(n + n_kv) * s:], stride, gu.i32_dev([0, b - a]), 1, b - a,
                                gu.i32_dev([a]), None, table, 100, s, 0, bt_dev, bt.shape[1], *pages, nb, kind, q_out[a:b])

    append(whole, 0, l)
    q_whole = q_out.clone()
    append(parts, 0, cut)
    append(parts, cut, l)
    torch.cuda.synchronize()
    for x, y in zip(whole, parts):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert torch.equal(q_whole, q_out)
    count = l - cut
    o = torch.empty(count, n, s, dtype=torch.bfloat16, device="cuda")
    ws = gu.workspace(ctx.ds_decode_window_workspace_bytes(count, l, window, sinks))
    ctx.ds_decode_attention_window(q_out[cut:], gu.i32_dev(np.arange(cut + 1, l + 1)), gu.i32_dev(np.repeat(bt, count, 0)), count,
                                   bt.shape[1], l, window, sinks, *parts, nb, kind, o, ws)
    torch.cuda.synchronize()
    kt = rwo.turned_bits(bits[1], rwo.angle_table(100, s)[:l], False)
    kk, vv = _stands(kt, kind), _stands(bits[2], kind)
    for i in range(count):
        end = cut + 1 + i
        want, pav, size, keys = rwo.attend_window(gu.to_f64(q_out[cut + i]), kk[:end], vv[:end], window, sinks)
        assert not close(gu.to_f64(o[i]), want, pav, size, s, keys)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_two_streams_at_once(gpu, kind):
    """Two contexts, each with its own stream and workspace, and a graph of each replayed beside the other's eager calls."""
    n, n_kv, s, window, sinks, B, l = 16, 2, 128, 700, 5, 3, 900
    kind, rng, stride = KINDS[kind], np.random.default_rng(5), (n + 2 * n_kv) * s
    table = torch.from_numpy(rwo.angle_table(l + 1, s)).cuda()
    cu = gu.i32_dev(synth.cu_seqlens([l] * B))

    class Side:
        def __init__(self):
            self.ctx = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)
            self.stream = torch.cuda.Stream()
            bt, self.nb = synth.make_block_tables([l + 1] * B, 16, 7)
            self.bt, self.width = gu.i32_dev(bt), bt.shape[1]
            self.pages = _pages(kind, self.nb, n_kv, s)
            self.flat, self.one = (gu.to_dev(np.concatenate([rows(rng, t, h, s) for h in (n, n_kv, n_kv)], 1).reshape(-1))
                                   for t in (B * l, B))
            self.q, self.k, self.o = (torch.empty(B * l, h, s, dtype=torch.bfloat16, device="cuda") for h in (n, n_kv, n))
            self.q1, self.o1 = (torch.empty(B, n, s, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.ws = gu.workspace(self.ctx.ds_decode_window_workspace_bytes(B, l + 1, window, sinks))
            self.lens = [gu.i32_dev([x] * B) for x in (0, l, l + 1)]

        def run(self):
            f, g, at = self.flat, self.one, ((n + n_kv) * s)
            self.ctx.ds_kv_append_rotary(f, stride, f[n * s:], f[at:], stride, cu, B, B * l, self.lens[0], None, table, l + 1, s,
                                         False, self.bt, self.width, *self.pages, self.nb, kind, self.q, self.k)
            self.ctx.ds_prefill_attention_window(self.q, n * s, self.k, n_kv * s, f[at:], stride, cu, B, B * l, l, window, sinks,
                                                 self.o)
            self.ctx.ds_kv_append_rotary(g, stride, g[n * s:], g[at:], stride, None, B, B, self.lens[1], None, table, l + 1, s,
                                         False, self.bt, self.width, *self.pages, self.nb, kind, self.q1)
            self.ctx.ds_decode_attention_window(self.q1, self.lens[2], self.bt, B, self.width, l + 1, window, sinks, *self.pages,
                                                self.nb, kind, self.o1, self.ws)

        def results(self):
            return [x.clone() for x in (self.q, self.k, self.o, self.q1, self.o1)]

    sides = [Side(), Side()]
    torch.cuda.synchronize()
    alone = []
    for x in sides:
        with torch.cuda.stream(x.stream):
            x.run()
        torch.cuda.synchronize()
        alone.append(x.results())
    graphs = []
    for x in sides:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=x.stream):
            x.run()
        graphs.append(graph)
    for turn in range(4):
        for x in sides:
            for y in (x.q, x.k, x.o, x.q1, x.o1):
                y.zero_()
        torch.cuda.synchronize()
        for i in (0, 1):
            with torch.cuda.stream(sides[i].stream):
                for _ in range(3):
                    graphs[i].replay() if turn % 2 == i else sides[i].run()
        torch.cuda.synchronize()
        for x, want in zip(sides, alone):
            assert all(torch.equal(a, b) for a, b in zip(x.results(), want)), turn
