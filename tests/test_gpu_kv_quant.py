"""The 8-bit cache as it is written and read back: every byte against the oracle's."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu
from tests.kv_pages import KINDS, Cache, rows, scales_dev, scales_host

pytestmark = pytest.mark.gpu

SHAPES = [(4, 4, 64), (8, 2, 128), (5, 5, 128), (3, 3, 64), (16, 1, 128), (40, 40, 128)]


def _ctx(n, n_kv, s):
    return binding.Context(n * s, n, s, 64, n_kv_heads=n_kv) if n * s % 64 == 0 else None


def _odd_rows(rng, t, n_kv, s):
    """Rows with what is hard: zeros, one number alone, ties, the least and the largest, infinities, NaN."""
    x = orc.from_bf16_bits(rows(rng, t, n_kv, s))
    specials = []
    z = np.zeros(s)
    specials.append(z.copy())
    for a in (1.0, 448.0, 450.0, 127.0, 254.0, 2.0 ** -133, 2.0 ** -120, 2.0 ** -92, 1.5 * 2.0 ** -95, 2.0 ** 127, 2.0 ** 100):
        y = z.copy()
        y[s // 3] = -a
        specials.append(y)
    y = rng.integers(-508, 509, s) / 4.0
    y[0] = 127.0
    specials.append(orc.from_bf16_bits(synth.f32_to_bf16_bits(y.astype(np.float32))))   # many halves of int8's steps
    y = rng.integers(-64, 65, s) * 7.0
    y[1] = -448.0
    specials.append(orc.from_bf16_bits(synth.f32_to_bf16_bits(y.astype(np.float32))))   # many halves of e4m3's steps
    y = rng.standard_normal(s)
    y[s - 1] = np.nan
    specials.append(y.copy())
    y[s - 1] = np.inf
    specials.append(y.copy())
    specials.append(np.full(s, -np.inf))
    flat = x.reshape(-1, s)
    at = rng.permutation(len(flat))[:len(specials)]
    for i, y in zip(at, specials):
        flat[i] = y
    with np.errstate(invalid="ignore"):
        return synth.f32_to_bf16_bits(flat.astype(np.float32)).reshape(t, n_kv, s)


def _poisoned(nb, n_kv, s):
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    k = torch.randint(0, 256, (nb, n_kv, 16, s), dtype=torch.uint8, device="cuda", generator=g)
    v = torch.randint(0, 256, (nb, n_kv, s, 16), dtype=torch.uint8, device="cuda", generator=g)
    sc = torch.randint(-2 ** 15, 2 ** 15, (2, nb, n_kv, 16), dtype=torch.int16, device="cuda", generator=g)
    return k, v, sc[0].view(torch.bfloat16), sc[1].view(torch.bfloat16)


def _expect(before, kind, k_bits, v_bits, lens, table, start=None):
    """What the pages are after the rows are written into them (start: positions of the rows, one a sequence)."""
    k, v, ks, vs = (before[0].cpu().numpy().copy(), before[1].cpu().numpy().copy(), gu.to_bits(before[2]).copy(),
                    gu.to_bits(before[3]).copy())
    kb, kc = kvo.quantise(orc.from_bf16_bits(k_bits), kind)
    vb, vc = kvo.quantise(orc.from_bf16_bits(v_bits), kind)
    kc, vc = gu.to_bits(scales_dev(kc)), gu.to_bits(scales_dev(vc))
    if start is None:
        kvo.to_pages(kb, kc, lens, table, k, ks, False)
        kvo.to_pages(vb, vc, lens, table, v, vs, True)
    else:
        for i, pos in enumerate(start):
            if pos >= 0:
                p, j = table[i][pos // 16], pos % 16
                k[p, :, j], v[p, :, :, j], ks[p, :, j], vs[p, :, j] = kb[i], vb[i], kc[i], vc[i]
    return k, v, ks, vs


def _same(after, want):
    torch.cuda.synchronize()
    got = (after[0].cpu().numpy(), after[1].cpu().numpy(), gu.to_bits(after[2]), gu.to_bits(after[3]))
    for name, g, w in zip(("k", "v", "k_scale", "v_scale"), got, want):
        bad = np.argwhere(g != w)
        assert not len(bad), (name, len(bad), bad[0], g[tuple(bad[0])], w[tuple(bad[0])])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s", SHAPES)
def test_hand_off_and_back(gpu, n, n_kv, s, kind):
    rng = np.random.default_rng(n * 1000 + s)
    ctx = _ctx(n, n_kv, s)
    for lens in ([1], [16], [17, 3, 32, 1], [100, 15, 33]):
        t, B, k = sum(lens), len(lens), KINDS[kind]
        k_bits, v_bits = _odd_rows(rng, t, n_kv, s), _odd_rows(rng, t, n_kv, s)
        table, nb = synth.make_block_tables([l + 20 for l in lens], 16, t)      # (more pages than the tokens need)
        before = _poisoned(nb, n_kv, s)
        after = tuple(x.clone() for x in before)
        cu, bt = gu.i32_dev(synth.cu_seqlens(lens)), gu.i32_dev(table)
        ctx.ds_kv_migrate_quant(gu.to_dev(k_bits), gu.to_dev(v_bits), cu, B, t, max(lens), bt, table.shape[1], *after, nb, k)
        want = _expect(before, k, k_bits, v_bits, lens, table)
        _same(after, want)
        # back: exactly what the bytes stand for, rounded once
        back = torch.full((2, t + 1, n_kv, s), 7.0, dtype=torch.bfloat16, device="cuda")
        ctx.ds_kv_read_quant(cu, B, t, max(lens), bt, table.shape[1], *after, nb, k, back[0], back[1])
        torch.cuda.synchronize()
        for got, bits in ((back[0], k_bits), (back[1], v_bits)):
            assert (got[t] == 7.0).all()
            stands = kvo.stands_for(*kvo.quantise(orc.from_bf16_bits(bits), k), k)
            most = 255 * 2.0 ** 120
            with np.errstate(invalid="ignore"):
                clipped = np.clip(stands, -most, most)
                rounded = synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(np.nan_to_num(clipped).astype(np.float32)))
            g = gu.to_f64(got[:t])
            np.testing.assert_array_equal(np.isnan(g), np.isnan(stands))
            np.testing.assert_array_equal(np.nan_to_num(g), np.where(np.isnan(stands), 0.0, rounded))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s", SHAPES)
def test_append(gpu, n, n_kv, s, kind):
    rng = np.random.default_rng(n * 77 + s)
    ctx, k = _ctx(n, n_kv, s), KINDS[kind]
    start = [0, 15, 16, 31, 5, -1, 100, 47, 3, 2, 1, 8, 9, 10, 11, 12, 13, 14, 6, 7]
    B, w = len(start), n_kv * s
    table, nb = synth.make_block_tables([max(p, 0) + 1 for p in start], 16, 3)
    before = _poisoned(nb, n_kv, s)
    bits = _odd_rows(rng, 2 * B, n_kv, s)
    for stride in (w, (n + 2 * n_kv) * s):                  # rows alone, or inside those of a QKV product
        buf = torch.full((B, stride + w), 5.0, dtype=torch.bfloat16, device="cuda").view(-1)[:B * stride + w]
        rows_k = torch.as_strided(buf, (B, w), (stride, 1), stride - w)
        gap = torch.full((B * stride + w,), 3.0, dtype=torch.bfloat16, device="cuda")
        rows_v = torch.as_strided(gap, (B, w), (stride, 1), 0)
        rows_k.copy_(gu.to_dev(bits[:B]).view(B, w))
        rows_v.copy_(gu.to_dev(bits[B:]).view(B, w))
        after = tuple(x.clone() for x in before)
        ctx.ds_kv_append_quant(rows_k, rows_v, stride, gu.i32_dev(start), gu.i32_dev(table), B, table.shape[1], *after, nb, k)
        _same(after, _expect(before, k, bits[:B], bits[B:], None, table, start))


def test_the_two_ways_of_writing_agree(gpu):
    """A prompt handed off whole, and its first part handed off and the rest appended token by token: the same bytes."""
    n, s, total, first = 8, 128, 45, 20
    rng = np.random.default_rng(9)
    ctx = _ctx(n, n, s)
    kb, vb = gu.to_dev(rows(rng, total, n, s)), gu.to_dev(rows(rng, total, n, s))
    table, nb = synth.make_block_tables([total], 16, 2)
    bt = gu.i32_dev(table)
    for kind in (binding.KV_E4M3, binding.KV_INT8):
        pages = []
        for upto in (total, first):
            p = _poisoned(nb, n, s)
            ctx.ds_kv_migrate_quant(kb, vb, gu.i32_dev([0, upto]), 1, upto, upto, bt, table.shape[1], *p, nb, kind)
            for j in range(upto, total):
                ctx.ds_kv_append_quant(kb[j], vb[j], n * s, gu.i32_dev([j]), bt, 1, table.shape[1], *p, nb, kind)
            pages.append(p)
        torch.cuda.synchronize()
        for a, b in zip(*pages):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_pages_behind_4_gib(gpu):
    """Page numbers whose bytes lie behind 32 bits' reach in K and in V."""
    n, s = 40, 128
    nb = 2 ** 32 // (n * 16 * s) + 40
    ctx = _ctx(n, n, s)
    rng = np.random.default_rng(1)
    lens = [33, 18]
    table = np.array([[nb - 1, 3, nb - 7], [nb - 2, nb - 3, -1]], np.int32)
    k = torch.empty((nb, n, 16, s), dtype=torch.uint8, device="cuda")
    v = torch.empty((nb, n, s, 16), dtype=torch.uint8, device="cuda")
    ks, vs = (torch.empty((nb, n, 16), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kb, vb = rows(rng, 51, n, s), rows(rng, 51, n, s)
    cu, bt = gu.i32_dev([0, 33, 51]), gu.i32_dev(table)
    kind = binding.KV_INT8
    ctx.ds_kv_migrate_quant(gu.to_dev(kb), gu.to_dev(vb), cu, 2, 51, 33, bt, 3, k, v, ks, vs, nb, kind)
    back = torch.empty((2, 51, n, s), dtype=torch.bfloat16, device="cuda")
    ctx.ds_kv_read_quant(cu, 2, 51, 33, bt, 3, k, v, ks, vs, nb, kind, back[0], back[1])
    q = gu.to_dev(rows(rng, 2, n, s))
    o = torch.empty_like(q)
    ws = gu.workspace(ctx.ds_decode_quant_workspace_bytes(2, 33))
    ctx.ds_decode_attention_quant(q, gu.i32_dev(lens), bt, 2, 3, 33, k, v, ks, vs, nb, kind, o, ws)
    torch.cuda.synchronize()
    used = np.concatenate([table[0], table[1][:2]])
    for page in used:                                       # (bytes of the pages, on the host one by one)
        assert torch.isfinite(ks[int(page)][:, :2].float()).all()
    for got, bits in ((back[0], kb), (back[1], vb)):
        stands = kvo.stands_for(*kvo.quantise(orc.from_bf16_bits(bits), kind), kind)
        np.testing.assert_array_equal(gu.to_bits(got), synth.f32_to_bf16_bits(stands.astype(np.float32)))
    a = 0
    for i, l in enumerate(lens):
        kk, vv = (kvo.stands_for(*kvo.quantise(orc.from_bf16_bits(b[a:a + l]), kind), kind) for b in (kb, vb))
        want, pav, size = kvo.attend(gu.to_f64(q[i]), kk, vv)
        assert (np.abs(gu.to_f64(o[i]) - want) <= kvo.attention_bound(want, pav, size, s, l)).all()
        a += l
