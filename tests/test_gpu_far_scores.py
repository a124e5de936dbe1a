"""Keys whose scores are below fp32's range, in chunks and tiles of nothing else: they weigh nothing, and the others what they
weigh without them.  Inputs are finite numbers throughout."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu
from tests.kv_pages import Cache, close

pytestmark = pytest.mark.gpu

FAR = 2.0 ** 60      # of a query's numbers; a key far off has -2^70: products of -2^130 and below, past -2^128


def _far(t):
    """Which of t tokens are far off: the first 128 of any 200, so whole chunks and tiles, and the last of all."""
    far = np.arange(t) % 200 < 128
    if t > 1:
        far[-1] = True
    return far


def _bits(x):
    return synth.f32_to_bf16_bits(x.astype(np.float32))


def _queries(rng, B, n, s):
    """All positive, so that no two products of a far key's score have unlike signs."""
    return _bits((1 + rng.random((B, n, s))) * FAR)


def _keys(rng, lens, n_kv, s):
    k = rng.standard_normal((sum(lens), n_kv, s)) / FAR / 2
    far = np.concatenate([_far(l) for l in lens])
    k[far] = -(1 + rng.random((int(far.sum()), n_kv, s))) * 2.0 ** 70
    return _bits(k)


def _cache(kind, lens, n_kv, s, seed):
    return Cache(kind, lens, n_kv, s, seed, k_bits=_keys(np.random.default_rng(seed), lens, n_kv, s))


def _check(got, q, parts, s):
    """parts: (k, v) of the row's keys, and which of them are far."""
    k, v, far = (np.concatenate(x) for x in zip(*parts))
    want, pav, size = kvo.attend(q, k[~far], v[~far])
    bad = close(got, want, pav, size, s, len(k))
    assert not bad, (len(k), int(far.sum()), bad)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s", [(4, 4, 64), (8, 2, 128), (40, 1, 128)])
@pytest.mark.parametrize("lens", [[150, 1, 64, 33, 400, 129], [3000]], ids=["short", "split"])
def test_own_pages(gpu, n, n_kv, s, lens, kind):
    c, B = _cache(kind, lens, n_kv, s, 3), len(lens)
    q = gu.to_dev(_queries(np.random.default_rng(1), B, n, s))
    ctx = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)
    o = torch.full_like(q, 9.0)
    ctx.ds_decode_attention_quant(q, gu.i32_dev(lens), gu.i32_dev(c.table), B, c.table.shape[1], max(lens), *c.args, o,
                                  gu.workspace(ctx.ds_decode_quant_workspace_bytes(B, max(lens))))
    torch.cuda.synchronize()
    for i, l in enumerate(lens):
        _check(gu.to_f64(o[i]), gu.to_f64(q[i]), [(*c.seq(i), _far(l))], s)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s,rows_of", [(4, 4, 64, [2, 1]), (8, 1, 128, [9, 1, 3]), (40, 1, 128, [1, 2]),
                                              (8, 8, 128, [20, 4])])
@pytest.mark.parametrize("prefix", [40, 2500], ids=["joined", "parts"])
def test_behind_prefixes(gpu, n, n_kv, s, rows_of, prefix, kind):
    groups, B = len(rows_of), sum(rows_of)
    plens = [prefix + 100 * g for g in range(groups)]
    own = [(67 * i) % 300 for i in range(B)]
    c = _cache(kind, plens + own, n_kv, s, 7)
    q = gu.to_dev(_queries(np.random.default_rng(2), B, n, s))
    ctx = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)
    cug = np.concatenate([[0], np.cumsum(rows_of)])
    o, pt, bt = torch.full_like(q, 9.0), gu.i32_dev(c.table[:groups]), gu.i32_dev(c.table[groups:])
    ctx.ds_decode_attention_shared(q, gu.i32_dev(cug), groups, max(rows_of), gu.i32_dev(plens), pt, pt.shape[1], max(plens),
                                   gu.i32_dev(own), bt, B, bt.shape[1], max(1, max(own)), *c.args, o,
                                   gu.workspace(ctx.ds_decode_shared_workspace_bytes(B, max(plens), max(1, max(own)))))
    torch.cuda.synchronize()
    for i in range(B):
        g = int(np.searchsorted(cug, i, side="right") - 1)
        _check(gu.to_f64(o[i]), gu.to_f64(q[i]), [(*c.seq(g), _far(plens[g])), (*c.seq(groups + i), _far(own[i]))], s)


@pytest.mark.parametrize("n,n_kv,s", [(4, 4, 64), (8, 2, 64), (8, 8, 128), (8, 2, 128), (40, 1, 128)])
@pytest.mark.parametrize("lens", [[150, 1, 64, 33, 400, 129], [3000]], ids=["short", "split"])
def test_the_bf16_cache(gpu, n, n_kv, s, lens):
    c, B = _cache("bf16", lens, n_kv, s, 3), len(lens)
    q = gu.to_dev(_queries(np.random.default_rng(1), B, n, s))
    ctx = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)
    o = torch.full_like(q, 9.0)
    ctx.ds_decode_attention(q, gu.i32_dev(lens), gu.i32_dev(c.table), B, c.table.shape[1], max(lens), c.k, c.v, c.nb, o,
                            gu.workspace(ctx.ds_decode_workspace_bytes(B, max(lens))))
    torch.cuda.synchronize()
    for i, l in enumerate(lens):
        _check(gu.to_f64(o[i]), gu.to_f64(q[i]), [(*c.seq(i), _far(l))], s)


@pytest.mark.parametrize("n,n_kv,s", [(4, 4, 64), (4, 2, 128)])
def test_prompts(gpu, n, n_kv, s):
    """Causal, over packed prompts; a query that sees far keys alone gets 0.  The sum counts the rounded probabilities here:
    2^-8 of the output more."""
    lens, rng = [400, 1, 129, 64, 150], np.random.default_rng(6)
    t = sum(lens)
    qb, kb, vb = _queries(rng, t, n, s), _keys(rng, lens, n_kv, s), _bits(rng.standard_normal((t, n_kv, s)))
    ctx = binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)
    q = gu.to_dev(qb)
    o = torch.full_like(q, 9.0)
    ctx.ds_prefill_attention(q, gu.to_dev(kb), gu.to_dev(vb), gu.i32_dev(synth.cu_seqlens(lens)), len(lens), t, max(lens), o)
    torch.cuda.synchronize()
    got, q, k, v, r0 = gu.to_f64(o), *(orc.from_bf16_bits(x) for x in (qb, kb, vb)), 0
    for l in lens:
        far = _far(l)
        for i in range(l):
            seen = np.flatnonzero(~far[:i + 1]) + r0
            want, pav, size = kvo.attend(q[r0 + i], k[seen], v[seen])
            bound = kvo.attention_bound(want, pav, size, s, i + 1) + 2.0 ** -8 * np.abs(want) * 1.01
            assert (np.abs(got[r0 + i] - want) <= bound).all(), (l, i)
        r0 += l


def test_nothing_but_far_keys_is_nothing(gpu):
    n, s, lens = 8, 128, [64, 5]
    k = -(1 + np.random.default_rng(0).random((69, n, s))) * 2.0 ** 70
    c = Cache("e4m3", lens, n, s, 4, k_bits=_bits(k))
    q = gu.to_dev(_queries(np.random.default_rng(1), 2, n, s))
    ctx, o = binding.Context(n * s, n, s, 64), torch.full_like(q, 9.0)
    ctx.ds_decode_attention_quant(q, gu.i32_dev(lens), gu.i32_dev(c.table), 2, c.table.shape[1], 64, *c.args, o,
                                  gu.workspace(ctx.ds_decode_quant_workspace_bytes(2, 64)))
    torch.cuda.synchronize()
    assert (o == 0).all()
