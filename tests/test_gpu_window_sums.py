"""Attention of prompts through a window divides by the sum of the very probabilities that it multiplies V with."""
import numpy as np
import pytest

from oracle import ds_oracle as orc
from paper_2401_09670_amd import synth
from tests import gpu_util as gu
from tests.kv_pages import rows
from tests.test_gpu_prefill_window import Call, _ctx

pytestmark = pytest.mark.gpu

# head size, sign of a, a, b of most keys and of one
FAR = [(64, 1, 2448, 18, 70), (64, -1, 2448, 122, 174), (128, 1, 2448, 50, 150), (128, -1, 2448, 148, 248)]


def _alike(rng, l, n_kv, s):
    """V of which every token is the same: bits [l, n_kv, s], nothing near 0."""
    c = rng.uniform(1, 2, (n_kv, s)) * np.where(rng.random((n_kv, s)) < 0.5, -1, 1) * 2.0 ** rng.integers(-6, 7, (n_kv, s))
    return np.ascontiguousarray(np.broadcast_to(synth.f32_to_bf16_bits(c.astype(np.float32)), (l, n_kv, s)))


# Weights that are rounded by d_j each make of a V that is c everywhere sum p_j (1 + d_j) c / sum p_j (1 + d_j) = c, whatever the
# d_j.  Products of two bf16 are exact in fp32; N terms of one sign lose at most N 2^-23 in either sum, a rescale 2^-24, the quotient
# and its product 2^-23: with N < 700 below 2^-12 in all, far less than the half step (2^-9 of a number at least) around c.
@pytest.mark.parametrize("spread", [0.05, 1.0, 4.0])
@pytest.mark.parametrize("n,n_kv,s", [(4, 4, 64), (8, 2, 64), (2, 2, 128), (16, 2, 128), (6, 2, 128)])
def test_a_v_that_is_the_same_everywhere_comes_back(gpu, n, n_kv, s, spread):
    ctx = _ctx(n, n_kv, s)
    for lens, window, sinks in (([300, 129, 1], 100, 4), ([200], 2, 1), ([70, 500], 600, 0)):
        rng = np.random.default_rng(sum(lens) + n)
        bits = [rows(rng, sum(lens), n, s, spread), rows(rng, sum(lens), n_kv, s), _alike(rng, sum(lens), n_kv, s)]
        c = Call(n, n_kv, s, lens, 1, bits=bits).run(ctx, window, sinks)
        want = np.repeat(bits[2], n // n_kv, axis=1)
        assert np.array_equal(gu.to_bits(c.o), want), (lens, window, sinks, (gu.to_bits(c.o) != want).mean())


@pytest.mark.parametrize("n,n_kv,s", [(4, 4, 64), (8, 2, 128)])
def test_rows_done_again_too(gpu, n, n_kv, s):
    """A NaN of one token and feature: rows that share a wave with it are done again, and nothing else of them changes."""
    l, window, sinks, at, f = 400, 30, 2, 210, 5
    rng = np.random.default_rng(2)
    bits = [rows(rng, l, n, s), rows(rng, l, n_kv, s), _alike(rng, l, n_kv, s)]
    want = np.repeat(bits[2], n // n_kv, axis=1)
    bits[2] = bits[2].copy()
    bits[2][at, :, f] = 0x7fc0
    got = gu.to_bits(Call(n, n_kv, s, [l], 1, bits=bits).run(_ctx(n, n_kv, s), window, sinks).o)
    i = np.arange(l)
    sees = (i >= at) & (i < at + window)
    assert (got[sees][:, :, f] & 0x7fff > 0x7f80).all()
    got[sees, :, f] = want[sees, :, f]
    assert np.array_equal(got, want), (got != want).mean()


def test_flat_scores_that_are_no_bf16_numbers(gpu):
    """The first 32 keys score a little less than all others, so that the others' probabilities lie between two bf16 numbers while the
    reference point stays: that they are all rounded alike does not move the result."""
    n, s, l = 2, 64, 320
    rng = np.random.default_rng(4)
    q, k = np.zeros((l, n, s), np.float32), np.zeros((l, n, s), np.float32)
    q[:, :, 0] = np.sqrt(s)
    # e^z 1 + 0.97 2^-8, a little less than half a step above 1, and 1.9 a quarter of a step from its neighbours
    for h, z in ((0, np.log1p(0.97 * 2.0 ** -8)), (1, np.log(1 + 115.25 * 2.0 ** -7))):
        k[32:, h, 0] = z
    v = 1.9 + 2.0 ** -7 * rng.standard_normal((l, n, s))
    bits = [synth.f32_to_bf16_bits(x.astype(np.float32)) for x in (q, k, v)]
    got = gu.to_f64(Call(n, n, s, [l], 1, bits=bits).run(_ctx(n, n, s), l, 0).o)
    qd, kd, vd = (orc.from_bf16_bits(b).astype(np.float64) for b in bits)
    for h in range(n):
        z = qd[:, h] @ kd[:, h].T / np.sqrt(s)
        p = np.where(np.arange(l) <= np.arange(l)[:, None], np.exp(z - z.max()), 0)
        p /= p.sum(1, keepdims=True)
        want = p @ vd[:, h]
        # sum p (1 + d) v / sum p (1 + d) - o = sum p d (v - o) / sum p (1 + d), |d| <= 2^-8; half a step of the result, which lies
        # between 1 and 2; scores off by 2^-22, sums of up to 400 terms in fp32
        away = (p[:, :, None] * np.abs(vd[None, :, h] - want[:, None])).sum(1)
        assert want.min() > 1 and want.max() < 2 - 2.0 ** -8
        bound = 2.0 ** -8 + 2.0 ** -8 * 1.01 * away + (2.0 ** -21 + 400 * 2.0 ** -23) * 2
        assert (np.abs(got[:, h] - want) <= bound).all(), (h, (np.abs(got[:, h] - want) / bound).max())


# Rows' scores are 2048 a + b or 2048 a + b / 2, exact in fp32, times log2(e) / sqrt(s) within 2^19 and 2^20: there a reference point is
# off by up to 2^-5 in the exponent, and from b = lower to b = upper by as much the other way.
@pytest.mark.parametrize("s,sign,a,lower,upper", FAR)
def test_equal_scores_on_either_side_of_another_reference_point(gpu, s, sign, a, lower, upper):
    """Keys of one score before and behind a key that moves the reference point weigh the same, in rows that it moves by more than the
    slack and in rows that it moves because another row of the wave is one of those."""
    n, l = 2, 64
    rng = np.random.default_rng(9)
    q, k = np.zeros((l, n, s), np.float32), np.zeros((l, n, s), np.float32)
    q[:, :, 0], q[::2, :, 1], q[1::2, :, 1] = 2048, 0.5, 1
    k[:, :, 0], k[:, :, 1] = sign * a, lower
    k[32, :, 1] = upper
    v = np.where(np.arange(l)[:, None, None] < 32, 1.5, -1.5) + 2.0 ** -5 * rng.standard_normal((l, n, s))
    v[32] *= 2.0 ** -8
    bits = [synth.f32_to_bf16_bits(x.astype(np.float32)) for x in (q, k, v)]
    qd, kd, vd = (orc.from_bf16_bits(b).astype(np.float64) for b in bits)
    assert (qd == q).all() and (kd == k).all()
    got = gu.to_f64(Call(n, n, s, [l], 1, bits=bits).run(_ctx(n, n, s), l, 0).o)
    for h in range(n):
        z = qd[:, h] @ kd[:, h].T
        z = (z - sign * 2048.0 * a) / np.sqrt(s)         # (what all of a row's scores have in common, taken off exactly)
        p = np.where(np.arange(l) <= np.arange(l)[:, None], np.exp(z - z.max(1, keepdims=True)), 0)
        p /= p.sum(1, keepdims=True)
        want = p @ vd[:, h]
        # The result's rounding; the probabilities' (2^-8 each), whose sum is that of the rounded ones; exponents of at most 24, their
        # scale and the exponentials in fp32, sums of 128 terms
        away = (p[:, :, None] * np.abs(vd[None, :, h] - want[:, None])).sum(1)
        bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * 1.01 * away + (2.0 ** -18 + 128 * 2.0 ** -23) * (p @ np.abs(vd[:, h]))
        worst = (np.abs(got[:, h] - want) / bound).max(1)
        assert (worst <= 1).all(), (h, worst.max(), worst.argmax())
