"""Decode attention through a sliding window with first tokens that stay visible, over pages of all three types, against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import kv_quant_oracle as kvo
from oracle import rotary_window_oracle as rwo
from paper_2401_09670_amd import binding
from tests import gpu_util as gu
from tests.kv_pages import Cache, close, rows

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "e4m3", "int8"]
# query heads, key/value heads, head size: as many, groups of 2 to 40, more queries than a tile or two have columns
SHAPES = [(4, 4, 64), (8, 2, 64), (40, 1, 64), (8, 8, 128), (16, 4, 128), (16, 1, 128), (17, 1, 128), (40, 1, 128)]
LENS = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 129, 255, 256, 257, 300]
WINDOWS = [(1, 0), (1, 1), (2, 16), (15, 4), (16, 4), (16, 0), (17, 33), (31, 17), (40, 64), (64, 0), (100, 5), (1, 128), (257, 4),
           (1000, 2000), (2 ** 31 - 1, 2 ** 31 - 1)]


def _ctx(n, n_kv, s):
    return binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)


def _given_back(c, window, sinks, lens=None):
    """The cache's pages with NaN in every slot that is hidden, and its table without the pages that hold nothing else."""
    k, v, table = c.k.clone(), c.v.clone(), c.table.copy()
    ks, vs = (None, None) if c.ks is None else (c.ks.clone(), c.vs.clone())
    at = []
    for i, l in enumerate(c.lens if lens is None else lens):
        see = np.zeros(16 * table.shape[1], bool)
        see[rwo.seen(l, window, sinks)] = True
        for p in range(table.shape[1]):
            if table[i, p] < 0:
                continue
            at += [(table[i, p], j) for j in range(16) if not see[16 * p + j]]
            if not see[16 * p:16 * p + 16].any():
                table[i, p] = -1
    if at:
        page, slot = (torch.tensor(x, device="cuda") for x in zip(*at))
        if ks is None:
            k[page, :, slot], v[page, :, slot] = float("nan"), float("nan")
        else:
            k[page, :, slot], v[page, :, :, slot] = 0x7f, 0x7f
            ks[page, :, slot], vs[page, :, slot] = float("nan"), float("nan")
    return table, (k, v, ks, vs, c.nb, c.kind)


def _attend(ctx, q, lens, table, pages, window, sinks, bound=None, ws=None):
    B, longest = len(lens), max(1, max(lens)) if bound is None else bound
    if ws is None:
        ws = gu.workspace(ctx.ds_decode_window_workspace_bytes(B, longest, window, sinks))
    o = torch.full_like(q, 9.0)
    ctx.ds_decode_attention_window(q, gu.i32_dev(lens), gu.i32_dev(table), B, table.shape[1], longest, window, sinks, *pages,
                                   o, ws)
    torch.cuda.synchronize()
    return o


def _check(o, q, c, s, window, sinks, lens=None, only=None):
    for i, l in enumerate(c.lens if lens is None else lens):
        if only is not None and i not in only:
            continue
        k, v = (x[:l] for x in c.seq(i))
        want, pav, size, keys = rwo.attend_window(gu.to_f64(q[i]), k, v, window, sinks)
        bad = close(gu.to_f64(o[i]), want, pav, size, s, keys)
        assert not bad, (i, l, window, sinks, bad)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,n_kv,s", SHAPES)
def test_lengths_and_windows(gpu, n, n_kv, s, kind):
    """Windows and first tokens that end anywhere in a page, meet, or hide nothing; what is hidden is NaN or not there."""
    c = Cache(kind, LENS, n_kv, s, seed=n + s, room=[l + 40 for l in LENS])
    q = gu.to_dev(rows(np.random.default_rng(n), len(LENS), n, s))
    ctx = _ctx(n, n_kv, s)
    for window, sinks in WINDOWS:
        _check(_attend(ctx, q, LENS, *_given_back(c, window, sinks), window, sinks), q, c, s, window, sinks)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,n_kv,s,lens,window,sinks", [
    (4, 4, 64, [5000], 3001, 4), (8, 1, 128, [6097, 2], 4000, 40), (40, 8, 128, [3001, 0, 2049], 2000, 0),
    (32, 1, 128, [7777, 900], 5000, 129), (8, 1, 128, [4000], 1600, 3000)])
def test_long_windows_split(gpu, n, n_kv, s, lens, window, sinks, kind):
    """Few rows: what is seen is split over workgroups, some of which have none of it."""
    c = Cache(kind, lens, n_kv, s, seed=3)
    q = gu.to_dev(rows(np.random.default_rng(2), len(lens), n, s))
    ctx = _ctx(n, n_kv, s)
    table, pages = _given_back(c, window, sinks)
    o = _attend(ctx, q, lens, table, pages, window, sinks)
    _check(o, q, c, s, window, sinks)
    # again, and with other numbers where the states go: the same bits
    size = ctx.ds_decode_window_workspace_bytes(len(lens), max(lens), window, sinks)
    assert size > 0
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(o, _attend(ctx, q, lens, table, pages, window, sinks, ws=ws))


@pytest.mark.parametrize("kind", KINDS)
def test_many_rows_of_unlike_lengths(gpu, kind):
    """Rows cut by how unequal what they see is, and more rows than a wave ranks at once."""
    n, n_kv, s, window, sinks = 16, 8, 64, 1800, 20
    rng = np.random.default_rng(0)
    lens = [int(x) for x in np.clip(rng.lognormal(6.0, 1.3, 100), 1, 5000)] + [4999, 5000]
    c = Cache(kind, lens, n_kv, s, seed=1)
    q = gu.to_dev(rows(np.random.default_rng(1), len(lens), n, s))
    ctx = _ctx(n, n_kv, s)
    table, pages = _given_back(c, window, sinks)
    only = set(np.argsort(lens)[-12:]) | set(range(10))
    _check(_attend(ctx, q, lens, table, pages, window, sinks), q, c, s, window, sinks, only=only)
    # a generous bound changes how it is cut alone
    wide = np.pad(table, ((0, 0), (0, 300)), constant_values=-1)
    _check(_attend(ctx, q, lens, wide, pages, window, sinks, bound=9000), q, c, s, window, sinks, only=only)


@pytest.mark.parametrize("kind", KINDS)
def test_a_window_that_hides_nothing_is_the_attention_without(gpu, kind):
    n, n_kv, s = 16, 4, 128
    lens = [70, 1, 300, 0, 16]
    c = Cache(kind, lens, n_kv, s, seed=5)
    q = gu.to_dev(rows(np.random.default_rng(3), len(lens), n, s))
    ctx = _ctx(n, n_kv, s)
    o = _attend(ctx, q, lens, c.table, c.args, 300, 0)
    assert torch.equal(o, _attend(ctx, q, lens, c.table, c.args, 1, 300))
    if kind != "bf16":
        want = torch.empty_like(o)
        ctx.ds_decode_attention_quant(q, gu.i32_dev(lens), gu.i32_dev(c.table), 5, c.table.shape[1], 300, *c.args, want,
                                      gu.workspace(ctx.ds_decode_quant_workspace_bytes(5, 300)))
        torch.cuda.synchronize()
        assert torch.equal(o, want)


def test_a_bound_below_a_length_drops_the_rest(gpu):
    n, s = 4, 64
    c = Cache("int8", [200, 90], n, s, seed=4)
    q = gu.to_dev(rows(np.random.default_rng(1), 2, n, s))
    o = _attend(_ctx(n, n, s), q, [200, 90], c.table, c.args, 30, 4, bound=120)
    _check(o, q, c, s, 30, 4, lens=[120, 90])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_a_row_that_is_not_finite(gpu, kind):
    """Seen, it makes NaN of the heads that see it; hidden, of nothing."""
    n, n_kv, s, lens, window, sinks = 8, 2, 128, [70, 70, 70, 70], 20, 3
    rng = np.random.default_rng(6)
    bits = {x: rows(rng, sum(lens), n_kv, s) for x in "kv"}
    bits["k"][2, 1, 5] = 0x7f80                 # sequence 0: the last of the first tokens, head 1
    bits["v"][70 + 3, 0, 0] = 0x7fc0            # sequence 1: hidden
    bits["v"][140 + 50, 0, 9] = 0xff80          # sequence 2: the window's first
    bits["k"][210 + 49, 1, 9] = 0xff80          # sequence 3: the last that is hidden
    c = Cache(kind, lens, n_kv, s, seed=2, k_bits=bits["k"], v_bits=bits["v"])
    q = gu.to_dev(rows(rng, 4, n, s))
    o = gu.to_f64(_attend(_ctx(n, n_kv, s), q, lens, c.table, c.args, window, sinks))
    nan = np.zeros((4, n), bool)
    nan[0, 4:], nan[2, :4] = True, True
    np.testing.assert_array_equal(np.isnan(o), np.broadcast_to(nan[..., None], o.shape))


@pytest.mark.parametrize("kind", KINDS)
def test_scores_below_the_range_weigh_nothing(gpu, kind):
    """Keys whose scores leave fp32's range downwards, in the window and among the first tokens: the others have all the
    weight; where there are no others, the output is 0."""
    n, s, lens, window, sinks = 2, 64, [40, 40], 10, 2
    k = np.zeros((80, n, s), np.float32)
    k[:40] = -3e38                              # sequence 0: all of them
    k[40:] = -3e38
    k[75] = 1.0                                 # sequence 1: but one in the window
    v = np.random.default_rng(3).standard_normal((80, n, s)).astype(np.float32)
    from paper_2401_09670_amd import synth
    c = Cache(kind, lens, n, s, seed=2, k_bits=synth.f32_to_bf16_bits(k), v_bits=synth.f32_to_bf16_bits(v))
    q = torch.full((2, n, s), 4.0, dtype=torch.bfloat16, device="cuda")
    o = gu.to_f64(_attend(_ctx(n, n, s), q, lens, c.table, c.args, window, sinks))
    assert (o[0] == 0).all()
    np.testing.assert_allclose(o[1], c.seq(1)[1][35], rtol=2.0 ** -8)


@pytest.mark.parametrize("kind", KINDS)
def test_captured_and_replayed_beside_another_graph(gpu, kind):
    """Two graphs on one workspace, replayed one after the other, lengths and queries changed between."""
    n, n_kv, s, window, sinks = 8, 2, 128, 1700, 20
    lens = [3000, 10, 1701]
    c = Cache(kind, lens, n_kv, s, seed=9)
    ctx, B = _ctx(n, n_kv, s), 3
    bt, kv = gu.i32_dev(c.table), gu.i32_dev(lens)
    ws = gu.workspace(ctx.ds_decode_window_workspace_bytes(B, 3000, window, sinks))
    q = [gu.to_dev(rows(np.random.default_rng(i), B, n, s)) for i in range(2)]
    o = [torch.zeros_like(x) for x in q]

    def call(i):
        ctx.ds_decode_attention_window(q[i], kv, bt, B, c.table.shape[1], 3000, (window, 500)[i], (sinks, 0)[i], *c.args, o[i],
                                       ws)

    for i in range(2):
        call(i)
    torch.cuda.synchronize()
    graphs, side = [torch.cuda.CUDAGraph() for _ in range(2)], torch.cuda.Stream()
    for i, g in enumerate(graphs):
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                call(i)
    for step in range(3):
        now = [3000 - 400 * step, 10 - step, 1701 - step]
        kv.copy_(gu.i32_dev(now))
        for i in range(2):
            q[i].copy_(gu.to_dev(rows(np.random.default_rng(10 + 2 * step + i), B, n, s)))
            o[i].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in o]
        for i in range(2):
            call(i)
            torch.cuda.synchronize()
            assert torch.equal(got[i], o[i])
            _check(got[i], q[i], c, s, (window, 500)[i], (sinks, 0)[i], lens=now)


@pytest.mark.parametrize("kind", KINDS)
def test_pages_behind_4_gib(gpu, kind):
    """A cache whose pages lie further behind its start than 32 bits reach."""
    n, n_kv, s, window, sinks = 16, 8, 128, 300, 20
    lens = [1000, 37]
    small = Cache(kind, lens, n_kv, s, seed=7)
    size = 2 if kind == "bf16" else 1
    far = (5 << 30) // (n_kv * 16 * s * size)
    nb = far + small.nb

    def behind(x):
        big = torch.empty((nb,) + tuple(x.shape[1:]), dtype=x.dtype, device="cuda")
        big[far:] = x
        return big

    pages = tuple(None if x is None else behind(x) for x in (small.k, small.v, small.ks, small.vs))
    table = np.where(small.table < 0, -1, small.table + far)
    q = gu.to_dev(rows(np.random.default_rng(4), 2, n, s))
    ctx = _ctx(n, n_kv, s)
    o = _attend(ctx, q, lens, table, (*pages, nb, small.kind), window, sinks)
    assert torch.equal(o, _attend(ctx, q, lens, small.table, small.args, window, sinks))
    _check(o, q, small, s, window, sinks)


def test_validation(gpu):
    n, s, lens, window, sinks = 4, 64, [100, 33], 20, 3
    c = Cache("int8", lens, n, s, seed=1)
    ctx = _ctx(n, n, s)
    ctx.ds_set_validate(True)
    q = gu.to_dev(rows(np.random.default_rng(4), 2, n, s))
    table, pages = _given_back(c, window, sinks)
    assert (table < 0).sum() > (c.table < 0).sum()
    _check(_attend(ctx, q, lens, table, pages, window, sinks), q, c, s, window, sinks)
    for seq, page in ((0, 0), (0, 5), (0, 6), (1, 0), (1, 1), (1, 2)):
        for wrong in (-1, c.nb):
            bad = table.copy()
            bad[seq, page] = wrong
            with pytest.raises(binding.DsError) as e:
                _attend(ctx, q, lens, bad, pages, window, sinks)
            assert e.value.status == 5
    for bad in ([100, -1], [101, 33]):
        with pytest.raises(binding.DsError) as e:
            _attend(ctx, q, bad, table, pages, window, sinks, bound=100)
        assert e.value.status == 5
