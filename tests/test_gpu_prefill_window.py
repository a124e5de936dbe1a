"""Attention of packed prompts through a sliding window with first tokens that stay visible, against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import rotary_window_oracle as rwo
from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu
from tests.kv_pages import rows

pytestmark = pytest.mark.gpu

# query heads, key/value heads, head size: as many, groups that are and are not powers of two, one key/value head for all
SHAPES = [(4, 4, 64), (8, 2, 64), (12, 4, 64), (2, 2, 128), (16, 2, 128), (6, 2, 128), (40, 1, 128), (32, 1, 64)]
LENS = [[1], [2, 1, 17], [64, 65, 63], [33, 128, 129, 5], [300]]
WINDOWS = [(1, 0), (1, 1), (2, 3), (16, 4), (17, 0), (32, 64), (40, 5), (64, 16), (65, 1), (100, 33), (129, 130), (500, 0),
           (2 ** 31 - 1, 2 ** 31 - 1)]


def _ctx(n, n_kv, s):
    return binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)


class Call:
    """Rows of a QKV product, `pad` elements between them, or Q, K and V by themselves."""

    def __init__(self, n, n_kv, s, lens, seed, pad=0, apart=False, extra=0, spread=1.0, bits=None):
        rng = np.random.default_rng(seed)
        self.n, self.n_kv, self.s, self.lens, self.t = n, n_kv, s, lens, sum(lens) + extra
        self.bits = [rows(rng, self.t, h, s, sp) for h, sp in ((n, spread), (n_kv, 1.0), (n_kv, 1.0))] if bits is None else bits
        if apart:
            self.q, self.k, self.v = (gu.to_dev(b) for b in self.bits)
            self.strides = n * s, n_kv * s, n_kv * s
        else:
            stride = (n + 2 * n_kv) * s + pad
            qkv = np.full((self.t, stride), 0x7fc1, np.uint16)
            qkv[:, :stride - pad] = np.concatenate(self.bits, 1).reshape(self.t, -1)
            flat = gu.to_dev(qkv).view(-1)
            self.q, self.k, self.v = flat, flat[n * s:], flat[(n + n_kv) * s:]
            self.strides = (stride,) * 3
        self.cu = gu.i32_dev(synth.cu_seqlens(lens))
        self.o = torch.full((self.t, n, s), 9.0, dtype=torch.bfloat16, device="cuda")

    def run(self, ctx, window, sinks, bound=None):
        self.o.fill_(9.0)
        (q, k, v), (a, b, c) = (self.q, self.k, self.v), self.strides
        ctx.ds_prefill_attention_window(q, a, k, b, v, c, self.cu, len(self.lens), self.t, bound or max(self.lens), window, sinks,
                                        self.o)
        torch.cuda.synchronize()
        return self

    def check(self, window, sinks, only=None, lens=None):
        got = gu.to_f64(self.o)
        q, k, v = (orc.from_bf16_bits(b) for b in self.bits)
        a = 0
        for l, upto in zip(self.lens, lens or self.lens):
            want, bound = attend(q[a:a + upto], k[a:a + upto], v[a:a + upto], window, sinks, only)
            at = np.arange(upto) if only is None else np.array([i for i in only if i < upto], int)
            bad = np.argwhere(~(np.abs(got[a + at] - want) <= bound))
            assert not len(bad), (window, sinks, l, at[bad[0][0]], bad[0], len(bad), got[a + at][tuple(bad[0])], want[tuple(bad[0])])
            assert (got[a + upto:a + l] == 9.0).all()
            a += l
        assert (got[a:] == 9.0).all()              # rows behind the last sequence


def attend(q, k, v, window, sinks, only=None):
    """[L, n, s] over [L, n_kv, s] in 64 bits, rows `only`, and how far a result may be from it: the result's own rounding
    (2^-8 of it); a probability's, 2^-8 of each in the numerator against the sum of the same rounded ones, so twice
    2^-8 sum p |v|; scores of s products in fp32, off by (s + 3) 2^-24 of sum |q_d k_d| / sqrt(s) each, the maximum's alike, and the
    exponent's rounding; sums over as many terms as there are keys."""
    L, n, s = q.shape
    g = n // k.shape[1]
    at = np.arange(L) if only is None else np.array([i for i in only if i < L], int)
    j = np.arange(L)
    see = (j <= at[:, None]) & ((at[:, None] - j < window) | (j < sinks))
    want, bound = np.zeros((len(at), n, s)), np.zeros((len(at), n, s))
    for h in range(n if len(at) else 0):
        kk, vv = k[:, h // g], v[:, h // g]
        z = np.where(see, q[at, h] @ kk.T / np.sqrt(s), -np.inf)
        size = np.where(see, np.abs(q[at, h]) @ np.abs(kk).T / np.sqrt(s), 0).max(1)
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        want[:, h] = p @ vv
        score = 2 * ((s + 3) * 2.0 ** -24 + 2.0 ** -23) * size
        rest = 2 * score + (see.sum(1) + 64) * 2.0 ** -23
        bound[:, h] = 2.0 ** -8 * np.abs(want[:, h]) * 1.01 + (2 * 2.0 ** -8 + rest[:, None]) * (p @ np.abs(vv)) * 1.01 + 1e-30
    return want, bound


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("n,n_kv,s", SHAPES)
def test_lengths_and_windows(gpu, n, n_kv, s, lens):
    ctx = _ctx(n, n_kv, s)
    for i, (window, sinks) in enumerate(WINDOWS):
        Call(n, n_kv, s, lens, n + s + i, pad=8 * (i % 3), apart=i % 2 == 1, extra=i % 4).run(ctx, window, sinks).check(window, sinks)


@pytest.mark.parametrize("n,n_kv,s,window,sinks", [(8, 1, 128, 700, 4), (2, 2, 128, 1024, 70), (4, 4, 64, 333, 0), (3, 1, 64, 2000, 9)])
def test_long_prompts(gpu, n, n_kv, s, window, sinks):
    rng = np.random.default_rng(5)
    only = sorted(set(rng.integers(0, 2500, 150)) | {0, 1, window - 1, window, window + 1, 2499, 2047, 2048})
    c = Call(n, n_kv, s, [2500, 40, 1200], 11).run(_ctx(n, n_kv, s), window, sinks)
    c.check(window, sinks, only=only)
    o = c.o.clone()
    assert torch.equal(o, c.run(_ctx(n, n_kv, s), window, sinks).o)     # the same bits


def test_many_sequences_some_empty(gpu):
    """More sequences than a wave looks through at once, lengths of 0 and 1 among them."""
    n, n_kv, s = 4, 2, 64
    rng = np.random.default_rng(6)
    lens = [int(x) for x in rng.integers(0, 40, 150)]
    Call(n, n_kv, s, lens, 7, extra=3).run(_ctx(n, n_kv, s), 9, 2).check(9, 2)


def test_steep_and_flat_scores(gpu):
    """Queries that pick one key of many, and queries that see all alike."""
    n, s = 4, 128
    for spread in (2.0 ** -20, 8.0):
        Call(n, n, s, [200, 77], 8, spread=spread).run(_ctx(n, n, s), 50, 3).check(50, 3)


@pytest.mark.parametrize("n,n_kv,s", [(8, 2, 64), (4, 4, 128)])
def test_a_window_that_hides_nothing_is_the_attention_without(gpu, n, n_kv, s):
    """Against the causal attention in the same bounds; and the two ways to see everything, bit by bit."""
    ctx, lens = _ctx(n, n_kv, s), [130, 1, 300]
    c = Call(n, n_kv, s, lens, 9, apart=True).run(ctx, 300, 0)
    c.check(300, 0)
    o = c.o.clone()
    assert torch.equal(o, c.run(ctx, 1, 300).o)
    want = torch.empty_like(o)
    ctx.ds_prefill_attention(c.q, c.k, c.v, c.cu, 3, c.t, 300, want)
    torch.cuda.synchronize()
    _, bound = zip(*[attend(*(orc.from_bf16_bits(b)[a:a + l] for b in c.bits), 300, 0) for a, l in ((0, 130), (130, 1), (131, 300))])
    assert (np.abs(gu.to_f64(o) - gu.to_f64(want)) <= 2 * np.concatenate(bound)).all()


@pytest.mark.parametrize("n,n_kv,s", [(8, 2, 64), (2, 2, 128), (16, 1, 128)])
def test_what_is_hidden_does_not_count(gpu, n, n_kv, s):
    """Infinities and NaN in K and V make NaN (or infinity) of the rows that see them, and of no other."""
    lens, window, sinks = [150, 90], 20, 3
    c = Call(n, n_kv, s, lens, 10)
    b = c.bits
    b[2][60, 0, 5], b[1][100, n_kv - 1, 7], b[2][1, 0, 9], b[2][150 + 40, 0, 0] = 0x7fc0, 0x7fc1, 0x7f80, 0xff80
    c = Call(n, n_kv, s, lens, 10, bits=b).run(_ctx(n, n_kv, s), window, sinks)
    got, g = gu.to_f64(c.o), n // n_kv
    i = np.arange(150)
    hit = np.zeros((240, n, s), bool)
    hit[:150][(i >= 60) & (i < 80), :g, 5] = True            # a NaN in V: that feature
    hit[:150][(i >= 100) & (i < 120), n - g:] = True         # in K: the row
    hit[:150][i >= 1, :g, 9] = True                          # an infinity of a first token
    hit[150:][(i[:90] >= 40) & (i[:90] < 60), :g, 0] = True
    assert not np.isfinite(got[hit]).any()
    assert np.isfinite(got[~hit]).all()
    clean = [np.where((x & 0x7f80) == 0x7f80, np.uint16(0), x) for x in b]
    q, k, v = (orc.from_bf16_bits(x) for x in clean)
    a = 0
    for l in lens:
        want, bound = attend(q[a:a + l], k[a:a + l], v[a:a + l], window, sinks)
        fine = ~hit[a:a + l]
        assert (np.abs(got[a:a + l] - want)[fine] <= bound[fine]).all()
        a += l


def test_scores_below_the_range_weigh_nothing(gpu):
    n, s = 2, 64
    k = np.zeros((60, n, s), np.float32)
    k[:] = -3e38
    k[50] = 1.0
    rng = np.random.default_rng(3)
    bits = [synth.f32_to_bf16_bits(x.astype(np.float32)) for x in (np.full((60, n, s), 4.0), k, rng.standard_normal((60, n, s)))]
    c = Call(n, n, s, [60], 1, bits=bits).run(_ctx(n, n, s), 5, 2)
    got, v = gu.to_f64(c.o), orc.from_bf16_bits(bits[2])
    assert (got[:50] == 0).all() and (got[55:] == 0).all()
    np.testing.assert_allclose(got[50:55], np.broadcast_to(v[50], (5, n, s)), rtol=2.0 ** -8)


@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 30, 2.0 ** 60])
def test_scores_far_from_zero(gpu, size):
    """Keys that are alike, but one of two heads' that is a step of bf16 larger: all weigh the same, or the one has all the weight,
    however far from 0 the scores are."""
    n, s, l, window, sinks = 2, 64, 150, 40, 3
    rng = np.random.default_rng(3)
    for sign in (1, -1):
        k = np.full((l, n, s), sign * size, np.float32)
        k[100, 1] *= 1 + sign * 2.0 ** -7
        bits = [synth.f32_to_bf16_bits(x.astype(np.float32)) for x in (np.ones((l, n, s)), k, rng.standard_normal((l, n, s)))]
        c = Call(n, n, s, [l], 1, bits=bits).run(_ctx(n, n, s), window, sinks)
        got, v = gu.to_f64(c.o), orc.from_bf16_bits(bits[2])
        for i in (0, 50, 99, 100, 120, 139, 140, 149):
            at = rwo.seen(i + 1, window, sinks)
            want, mean = v[at].mean(0), np.abs(v[at]).mean(0)
            if 100 <= i < 140:
                want[1], mean[1] = v[100, 1], np.abs(v[100, 1])
            # weights that are equal: their rounding to bf16 is too; sums in fp32, the quotient, the result's rounding
            assert (np.abs(got[i] - want) <= 2.0 ** -8 * np.abs(want) * 1.01 + 2 * (2.0 ** -8 + 100 * 2.0 ** -23) * mean).all(), (size, i)


def test_nothing_finite_at_all(gpu):
    """NaN and infinities in all of V take longer and make NaN of all that is seen."""
    n, n_kv, s, l = 16, 2, 128, 3000
    rng = np.random.default_rng(4)
    bits = [rows(rng, l, h, s) for h in (n, n_kv, n_kv)]
    bits[2][:] = 0x7fc0
    bits[2][::3] = 0x7f80
    c = Call(n, n_kv, s, [l - 7, 7], 1, bits=bits).run(_ctx(n, n_kv, s), 500, 4)
    assert torch.isnan(c.o.float()).all()


@pytest.mark.parametrize("s", [64, 128])
def test_a_hidden_nan_of_any_feature(gpu, s):
    """One feature of one token's V: nothing of the rows that do not see it changes, whichever feature it is."""
    n, n_kv, l, window, at = 2, 1, 70, 10, 30
    rng = np.random.default_rng(8)
    bits = [rows(rng, l, h, s) for h in (n, n_kv, n_kv)]
    ctx = _ctx(n, n_kv, s)
    clean = gu.to_f64(Call(n, n_kv, s, [l], 1, bits=bits).run(ctx, window, 1).o)
    i = np.arange(l)
    sees = (i >= at) & (i < at + window)
    for f in range(s):
        spoilt = [bits[0], bits[1], bits[2].copy()]
        spoilt[2][at, 0, f] = 0x7fc0
        got = gu.to_f64(Call(n, n_kv, s, [l], 1, bits=spoilt).run(ctx, window, 1).o)
        assert np.isnan(got[sees][:, :, f]).all(), f
        got[sees, :, f] = clean[sees, :, f]
        # Done again or not, a result is off by its rounding and its probabilities' (attend): 3 * 2^-8 of the largest V and the
        # little that scores and sums lose; and there are two.
        assert (np.abs(got - clean) <= 2.0 ** -5 * np.abs(gu.to_f64(gu.to_dev(bits[2]))).max()).all(), f


@pytest.mark.parametrize("s", [64, 128])
def test_an_infinity_that_all_see(gpu, s):
    """Of V: NaN of the feature in every row that sees it, whether or not another row of the wave does not."""
    n, n_kv, l = 4, 2, 140
    rng = np.random.default_rng(6)
    bits = [rows(rng, l, h, s) for h in (n, n_kv, n_kv)]
    bits[2][0, 0, 3], bits[2][0, 1, s - 1] = 0x7f80, 0xff80
    for window, sinks in ((200, 0), (5, 1)):
        got = gu.to_f64(Call(n, n_kv, s, [l], 1, bits=bits).run(_ctx(n, n_kv, s), window, sinks).o)
        hit = np.zeros((l, n, s), bool)
        hit[:, :2, 3] = hit[:, 2:, s - 1] = True
        assert np.isnan(got[hit]).all() and np.isfinite(got[~hit]).all()


def test_a_bound_below_a_length_drops_the_rest(gpu):
    n, s = 4, 64
    Call(n, n, s, [200, 90], 4).run(_ctx(n, n, s), 30, 4, bound=120).check(30, 4, lens=[120, 90])


def test_rows_behind_4_gib(gpu):
    """Rows whose bytes lie further from the first than 32 bits reach."""
    n, n_kv, s, stride, lens = 16, 2, 128, 2 ** 18, [8950, 100]
    small = Call(n, n_kv, s, lens, 12, apart=True)
    big = torch.zeros(small.t, stride, dtype=torch.bfloat16, device="cuda")
    flat = big.view(-1)
    for b, x in ((0, small.q), (n * s, small.k), ((n + n_kv) * s, small.v)):
        big[:, b:b + x[0].numel()] = x.flatten(1)
    assert big.numel() * 2 > 2 ** 32
    ctx = _ctx(n, n_kv, s)
    small.run(ctx, 100, 4)
    o = torch.zeros_like(small.o)
    ctx.ds_prefill_attention_window(flat, stride, flat[n * s:], stride, flat[(n + n_kv) * s:], stride, small.cu, 2, small.t, 8950,
                                    100, 4, o)
    torch.cuda.synchronize()
    assert torch.equal(o, small.o)
    small.check(100, 4, only=list(range(8900, 8950)) + [0, 1, 99])


def test_captured_and_replayed(gpu):
    """A graph on a stream of its own, inputs and lengths changed between the replays."""
    n, n_kv, s = 8, 2, 128
    ctx = _ctx(n, n_kv, s)
    c = Call(n, n_kv, s, [100, 60], 13)
    c.run(ctx, 33, 4, bound=160)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            ctx.ds_prefill_attention_window(c.q, c.strides[0], c.k, c.strides[1], c.v, c.strides[2], c.cu, 2, c.t, 160, 33, 4, c.o)
    for step, lens in enumerate(([100, 60], [1, 159], [60, 40])):
        other = Call(n, n_kv, s, lens, 20 + step, extra=160 - sum(lens))
        c.q.copy_(other.q)
        c.cu.copy_(other.cu)
        c.o.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        other.o = c.o
        other.check(33, 4)


def test_validation(gpu):
    n, s = 4, 64
    ctx = _ctx(n, n, s)
    ctx.ds_set_validate(True)
    c = Call(n, n, s, [20, 13], 4)
    c.run(ctx, 5, 1).check(5, 1)
    for cu in ([1, 20, 33], [0, 20, 32], [0, 33, 33], [0, 34, 33]):
        c.cu = gu.i32_dev(cu)
        with pytest.raises(binding.DsError) as e:
            c.run(ctx, 5, 1)
        assert e.value.status == 5
