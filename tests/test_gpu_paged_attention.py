"""Decode attention over the 8-bit cache, and behind prefixes that rows share, against 64 bits on what the pages hold."""
import numpy as np
import pytest
import torch

from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import binding
from tests import gpu_util as gu
from tests.kv_pages import Cache, close, rows

pytestmark = pytest.mark.gpu

# query heads, key/value heads, head size: as many, groups of 2 to 40, more queries than a tile or two have columns
SHAPES = [(4, 4, 64), (8, 2, 64), (40, 1, 64), (8, 8, 128), (16, 4, 128), (16, 1, 128), (17, 1, 128), (40, 1, 128)]
LENS = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 129, 255, 256, 257, 300]


def _ctx(n, n_kv, s):
    return binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)


def _attend(ctx, q, c, lens=None, room=None, max_len=None):
    lens = c.lens if lens is None else lens
    B, longest = len(lens), max(1, max(lens)) if max_len is None else max_len
    ws = gu.workspace(ctx.ds_decode_quant_workspace_bytes(B, longest) if room is None else room)
    o = torch.full_like(q, 9.0)
    ctx.ds_decode_attention_quant(q, gu.i32_dev(lens), gu.i32_dev(c.table), B, c.table.shape[1], longest, *c.args, o, ws)
    torch.cuda.synchronize()
    return o


def _check(o, q, c, n, s, lens=None):
    for i, l in enumerate(c.lens if lens is None else lens):
        k, v = (x[:l] for x in c.seq(i))
        want, pav, size = kvo.attend(gu.to_f64(q[i]), k, v)
        bad = close(gu.to_f64(o[i]), want, pav, size, s, l)
        assert not bad, (i, l, bad)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s", SHAPES)
def test_lengths(gpu, n, n_kv, s, kind):
    c = Cache(kind, LENS, n_kv, s, seed=n + s, room=[l + 40 for l in LENS])
    q = gu.to_dev(rows(np.random.default_rng(n), len(LENS), n, s))
    _check(_attend(_ctx(n, n_kv, s), q, c), q, c, n, s)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s,lens", [(4, 4, 64, [5000]), (8, 1, 128, [4097, 2]), (40, 8, 128, [1, 0, 2049])])
def test_long_ones_split(gpu, n, n_kv, s, lens, kind):
    """Few rows: the pages are split over workgroups, some of which have none."""
    c = Cache(kind, lens, n_kv, s, seed=3)
    q = gu.to_dev(rows(np.random.default_rng(2), len(lens), n, s))
    ctx = _ctx(n, n_kv, s)
    o = _attend(ctx, q, c)
    _check(o, q, c, n, s)
    # again, and with other numbers where the states go: the same bits
    assert torch.equal(o, _attend(ctx, q, c))
    ws = torch.full((ctx.ds_decode_quant_workspace_bytes(len(lens), max(lens)),), 255, dtype=torch.uint8, device="cuda")
    o2 = torch.empty_like(o)
    ctx.ds_decode_attention_quant(q, gu.i32_dev(lens), gu.i32_dev(c.table), len(lens), c.table.shape[1], max(lens), *c.args,
                                  o2, ws)
    torch.cuda.synchronize()
    assert torch.equal(o, o2)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_steep_and_flat_scores(gpu, kind):
    """Queries that pick one key of many, and queries that see all alike."""
    n, s = 8, 128
    for spread in (2.0 ** -20, 6.0):
        c = Cache(kind, [300, 77], n, s, seed=8, spread=spread)
        q = gu.to_dev(rows(np.random.default_rng(5), 2, n, s, 4.0))
        _check(_attend(_ctx(n, n, s), q, c), q, c, n, s)


def test_many_rows(gpu):
    n, n_kv, s = 16, 2, 128
    lens = list(np.random.default_rng(0).integers(1, 200, 150))
    c = Cache("e4m3", lens, n_kv, s, seed=1)
    q = gu.to_dev(rows(np.random.default_rng(1), len(lens), n, s))
    _check(_attend(_ctx(n, n_kv, s), q, c), q, c, n, s)


def test_shorter_than_what_the_cache_holds(gpu):
    """kv_lens says how many of the tokens count; a larger bound than any of them changes the splits alone."""
    n, s = 4, 64
    c = Cache("int8", [200, 200], n, s, seed=4)
    q = gu.to_dev(rows(np.random.default_rng(1), 2, n, s))
    _check(_attend(_ctx(n, n, s), q, c, lens=[30, 161], max_len=200), q, c, n, s, lens=[30, 161])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("where", ["k", "v"])
def test_a_row_that_is_not_finite(gpu, kind, where):
    """It makes NaN of the heads that see it, in every split that is merged, and of nothing else."""
    n, n_kv, s = 8, 2, 128
    lens = [1, 70, 1500, 70]
    rng = np.random.default_rng(6)
    bits = {x: rows(rng, sum(lens), n_kv, s) for x in "kv"}
    bits[where][0, 1, 5] = 0x7f80               # sequence 0, its only token, key/value head 1
    bits[where][1 + 69, 0, 0] = 0x7fc0          # sequence 1, its last token, head 0
    bits[where][71 + 800, 1, 127] = 0xff80      # sequence 2, in the middle, head 1
    c = Cache(kind, lens, n_kv, s, seed=2, k_bits=bits["k"], v_bits=bits["v"])
    q = gu.to_dev(rows(rng, 4, n, s))
    o = gu.to_f64(_attend(_ctx(n, n_kv, s), q, c))
    nan = np.zeros((4, n), bool)
    nan[0, 4:], nan[1, :4], nan[2, 4:] = True, True, True
    np.testing.assert_array_equal(np.isnan(o), np.broadcast_to(nan[..., None], o.shape))
    for i, l in enumerate(lens):
        k, v = c.seq(i)
        with np.errstate(invalid="ignore"):
            want, pav, size = kvo.attend(gu.to_f64(q[i]), k, v)
        fine = ~nan[i]
        assert not close(o[i][fine], want[fine], pav[fine], size[fine], s, l)


def _groups(rows_of, prefix, own, n_kv, s, kind, seed):
    """One cache whose first sequences are the groups' prefixes, the others the rows' own tokens."""
    c = Cache(kind, list(prefix) + list(own), n_kv, s, seed)
    return c, np.concatenate([[0], np.cumsum(rows_of)])


def _shared(ctx, q, c, cu, prefix, own, room=None, slack=0):
    g, B = len(prefix), len(own)
    mr, mp, mk = int(np.diff(cu).max()), max(1, max(prefix)) + slack, max(1, max(own)) + slack
    pt, bt = c.table[:g], c.table[g:]
    if slack:
        pt, bt = (np.pad(x, ((0, 0), (0, -(-slack // 16))), constant_values=-1) for x in (pt, bt))
    ws = gu.workspace(ctx.ds_decode_shared_workspace_bytes(B, mp, mk) if room is None else room)
    o = torch.full_like(q, 9.0)
    ctx.ds_decode_attention_shared(q, gu.i32_dev(cu), g, mr, gu.i32_dev(prefix), gu.i32_dev(pt), pt.shape[1], mp,
                                   gu.i32_dev(own), gu.i32_dev(bt), B, bt.shape[1], mk, *c.args, o, ws)
    torch.cuda.synchronize()
    return o


def _check_shared(o, q, c, cu, s):
    g = len(cu) - 1
    for j in range(g):
        kp, vp = c.seq(j)
        for i in range(cu[j], cu[j + 1]):
            k, v = c.seq(g + i)
            k, v = np.concatenate([kp, k]), np.concatenate([vp, v])
            want, pav, size = kvo.attend(gu.to_f64(q[i]), k, v)
            bad = close(gu.to_f64(o[i]), want, pav, size, s, len(k))
            assert not bad, (j, i, len(kp), len(k), bad)


GROUPS = [
    ([3], [45], [0, 1, 20]),                                  # a prefix that ends inside a page
    ([2, 1, 4], [16, 0, 33], [5, 0, 0, 17, 1, 64, 16]),       # one without a prefix, one row without anything
    ([1, 0, 2], [100, 70, 1], [3, 40, 0]),                    # a group without rows
    ([7], [700], [1, 2, 3, 4, 5, 6, 7]),
    ([1, 1], [64, 63], [0, 0]),                               # nothing but the prefix
]


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s", SHAPES)
def test_shared_prefixes(gpu, n, n_kv, s, kind):
    ctx = _ctx(n, n_kv, s)
    for seed, (rows_of, prefix, own) in enumerate(GROUPS):
        c, cu = _groups(rows_of, prefix, own, n_kv, s, kind, seed)
        q = gu.to_dev(rows(np.random.default_rng(seed), len(own), n, s))
        o = _shared(ctx, q, c, cu, prefix, own)
        _check_shared(o, q, c, cu, s)
        assert torch.equal(o, _shared(ctx, q, c, cu, prefix, own))


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s,B", [(4, 4, 64, 70), (8, 8, 128, 33), (16, 2, 128, 40), (8, 2, 64, 130)])
def test_wide_groups(gpu, n, n_kv, s, B, kind):
    """More queries of a key/value head than a workgroup has columns, the last ones not full."""
    rng = np.random.default_rng(B)
    own = list(rng.integers(0, 40, B))
    rows_of = [B - 5, 5]
    c, cu = _groups(rows_of, [333, 18], own, n_kv, s, kind, 1)
    q = gu.to_dev(rows(rng, B, n, s))
    ctx = _ctx(n, n_kv, s)
    _check_shared(_shared(ctx, q, c, cu, [333, 18], own), q, c, cu, s)
    # larger bounds than what is there: other splits, the same values
    _check_shared(_shared(ctx, q, c, cu, [333, 18], own, slack=1000), q, c, cu, s)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_long_prefix(gpu, kind):
    n, n_kv, s = 8, 2, 128
    own = [9, 0, 30]
    c, cu = _groups([3], [6001], own, n_kv, s, kind, 7)
    q = gu.to_dev(rows(np.random.default_rng(3), 3, n, s))
    _check_shared(_shared(_ctx(n, n_kv, s), q, c, cu, [6001], own), q, c, cu, s)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
def test_a_prefix_that_is_not_finite(gpu, kind):
    """NaN for the rows of its group, at the heads that see it."""
    n, s = 4, 64
    rng = np.random.default_rng(3)
    prefix, own = [50, 50], [10, 20, 30]
    t = sum(prefix) + sum(own)
    kb, vb = rows(rng, t, n, s), rows(rng, t, n, s)
    vb[49, 2, 7] = 0x7fc0
    c = Cache(kind, prefix + own, n, s, 5, k_bits=kb, v_bits=vb)
    q = gu.to_dev(rows(rng, 3, n, s))
    o = gu.to_f64(_shared(_ctx(n, n, s), q, c, np.array([0, 2, 3]), prefix, own))
    # (of bf16 pages the one feature alone: a row there has no scale that is shared)
    nan = np.zeros(o.shape, bool)
    if kind == "bf16":
        nan[:2, 2, 7] = True
    else:
        nan[:2, 2] = True
    np.testing.assert_array_equal(np.isnan(o), nan)


def test_graph_replays_and_another_stream(gpu):
    """Both attentions and both writes of a step captured on a side stream, replayed after the inputs changed, against the
    same calls run eagerly."""
    n, n_kv, s = 8, 2, 128
    ctx = _ctx(n, n_kv, s)
    kind, prefix, own = "int8", [90, 40], [10, 33, 64, 1]
    c = Cache(kind, prefix + own, n_kv, s, 3, room=prefix + [o + 4 for o in own])
    cu = np.array([0, 3, 4])
    rng = np.random.default_rng(0)
    q, kn, vn = (gu.to_dev(rows(rng, 4, h, s)) for h in (n, n_kv, n_kv))
    lens, pt, bt = gu.i32_dev(own), gu.i32_dev(c.table[:2]), gu.i32_dev(c.table[2:])
    kv_lens = gu.i32_dev([l + 1 for l in own])
    cud, pl = gu.i32_dev(cu), gu.i32_dev(prefix)
    mb, longest = c.table.shape[1], max(own) + 4
    ws = gu.workspace(max(ctx.ds_decode_shared_workspace_bytes(4, 90, longest), ctx.ds_decode_quant_workspace_bytes(4, longest)))
    pages = [x.clone() for x in (c.k, c.v, c.ks, c.vs)]
    o1, o2 = torch.empty_like(q), torch.empty_like(q)

    def step(p, a, b):
        ctx.ds_kv_append_quant(kn, vn, n_kv * s, lens, bt, 4, mb, *p, c.nb, c.kind)
        ctx.ds_decode_attention_quant(q, kv_lens, bt, 4, mb, longest, *p, c.nb, c.kind, a, ws)
        ctx.ds_decode_attention_shared(q, cud, 2, 3, pl, pt, mb, 90, kv_lens, bt, 4, mb, longest, *p, c.nb, c.kind, b, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step([x.clone() for x in pages], torch.empty_like(q), torch.empty_like(q))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(pages, o1, o2)
    for i in range(3):
        q.copy_(gu.to_dev(rows(rng, 4, n, s)))
        kn.copy_(gu.to_dev(rows(rng, 4, n_kv, s)))
        eager = [x.clone() for x in pages]
        e1, e2 = torch.empty_like(q), torch.empty_like(q)
        graph.replay()
        torch.cuda.synchronize()
        step(eager, e1, e2)
        torch.cuda.synchronize()
        assert torch.equal(o1, e1) and torch.equal(o2, e2), i
        for a, b in zip(pages, eager):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
        lens += 1               # the next token, behind the one that was just appended
        kv_lens += 1


def test_the_least_workspace_serves_and_less_is_refused(gpu):
    n, n_kv, s = 8, 1, 128
    ctx = _ctx(n, n_kv, s)
    c = Cache("e4m3", [2000, 30], n_kv, s, 1)
    q = gu.to_dev(rows(np.random.default_rng(0), 2, n, s))
    args = (q, gu.i32_dev(c.lens), gu.i32_dev(c.table), 2, c.table.shape[1], 2000, *c.args)
    o = torch.empty_like(q)
    with pytest.raises(binding.DsError) as e:
        ctx.ds_decode_attention_quant(*args, o, None)
    need = int(str(e.value).split("<")[1])
    assert 0 < need <= ctx.ds_decode_quant_workspace_bytes(2, 2000)
    with pytest.raises(binding.DsError):
        ctx.ds_decode_attention_quant(*args, o, torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    guarded = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    ctx.ds_decode_attention_quant(*args, o, guarded[:need])
    torch.cuda.synchronize()
    assert (guarded[need:] == 171).all()
    _check(o, q, c, n, s)
