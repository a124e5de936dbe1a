"""How many bits the probabilities keep in the second product of the attention over pages: 16 (two bf16 numbers each), so that
what is left of an output's error is its own rounding to bf16, also where terms of unlike signs cancel.  Not asked of wide tiles
over 8 bits (more than 16 columns), where a probability is one bf16 number."""
import numpy as np
import pytest
import torch

from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import binding
from tests import gpu_util as gu
from tests.kv_pages import Cache, rows

pytestmark = pytest.mark.gpu


def _bound(o, p_abs_v, size, s, keys):
    """As kv_quant_oracle.attention_bound, but for the probabilities: near = a bf16 within 2^-8 of p, rest = a bf16 within 2^-8
    of p - near (exact in fp32), so near + rest is within 2^-16 of p, and 2^-16 sum p |v| takes the place of 2^-8 sum p |v|."""
    score = 2 * ((s + 3) * 2.0 ** -24 + 2.0 ** -23) * size
    rest = 2 * score + (keys + 64) * 2.0 ** -23
    return 2.0 ** -8 * np.abs(o) * 1.01 + (2.0 ** -16 + rest[..., None]) * p_abs_v * 1.01 + 1e-30


def _check(got, q, k, v, s):
    want, pav, size = kvo.attend(gu.to_f64(q), k, v)
    over = np.abs(gu.to_f64(got) - want) / _bound(want, pav, size, s, len(k))
    assert over.max(initial=0) <= 1, (len(k), over.max())


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s,lens", [
    (4, 4, 64, [300, 17, 1, 64]), (8, 2, 128, [300, 17, 1, 64]), (16, 1, 128, [257, 40]),
    (4, 4, 64, [3000]), (8, 1, 128, [5000, 2]),                 # split
    (40, 40, 128, [30 + i % 200 for i in range(40)]),           # a wave a head
])
def test_own_pages_of_8_bits(gpu, n, n_kv, s, lens, kind):
    c, B = Cache(kind, lens, n_kv, s, 5), len(lens)
    q = gu.to_dev(rows(np.random.default_rng(3), B, n, s))
    ctx, o = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv), torch.full_like(q, 9.0)
    ctx.ds_decode_attention_quant(q, gu.i32_dev(lens), gu.i32_dev(c.table), B, c.table.shape[1], max(lens), *c.args, o,
                                  gu.workspace(ctx.ds_decode_quant_workspace_bytes(B, max(lens))))
    torch.cuda.synchronize()
    for i in range(B):
        _check(o[i], q[i], *c.seq(i), s)


@pytest.mark.parametrize("kind,n,n_kv,s,rows_of", [
    ("bf16", 4, 4, 64, [2, 3]), ("bf16", 8, 2, 128, [3, 1]), ("e4m3", 8, 8, 128, [3, 2]), ("int8", 8, 2, 128, [2, 4]),
    ("bf16", 8, 8, 128, [20, 4]), ("bf16", 16, 2, 64, [1, 9, 3]), ("bf16", 40, 1, 128, [1, 2]),   # wide
])
@pytest.mark.parametrize("prefix", [40, 1500], ids=["joined", "parts"])
def test_behind_prefixes(gpu, kind, n, n_kv, s, rows_of, prefix):
    groups, B = len(rows_of), sum(rows_of)
    plens, own = [prefix + 50 * g for g in range(groups)], [(37 * i) % 120 for i in range(B)]
    c = Cache(kind, plens + own, n_kv, s, 8)
    q = gu.to_dev(rows(np.random.default_rng(4), B, n, s))
    ctx, o = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv), torch.full_like(q, 9.0)
    cug = np.concatenate([[0], np.cumsum(rows_of)])
    pt, bt = gu.i32_dev(c.table[:groups]), gu.i32_dev(c.table[groups:])
    ctx.ds_decode_attention_shared(q, gu.i32_dev(cug), groups, max(rows_of), gu.i32_dev(plens), pt, pt.shape[1], max(plens),
                                   gu.i32_dev(own), bt, B, bt.shape[1], max(own), *c.args, o,
                                   gu.workspace(ctx.ds_decode_shared_workspace_bytes(B, max(plens), max(own))))
    torch.cuda.synchronize()
    for i in range(B):
        g = int(np.searchsorted(cug, i, side="right") - 1)
        (kp, vp), (k, v) = c.seq(g), c.seq(groups + i)
        _check(o[i], q[i], np.concatenate([kp, k]), np.concatenate([vp, v]), s)
