"""The oracle of rotated positions and windows: hand values, complex numbers, masks written out, torch's softmax."""
import math

import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import rotary_window_oracle as rwo
from paper_2401_09670_amd import synth


def test_table():
    t = rwo.angle_table(50, 8, base=100.0)
    assert t.dtype == np.float32 and t.shape == (50, 8)
    np.testing.assert_array_equal(t[0], [1, 1, 1, 1, 0, 0, 0, 0])
    for p in (1, 7, 49):
        for i in range(4):
            angle = p * 100.0 ** (-2 * i / 8)
            # the nearest fp32
            assert abs(t[p, i] - math.cos(angle)) <= 2.0 ** -24 and abs(t[p, 4 + i] - math.sin(angle)) <= 2.0 ** -24


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("rot,s", [(16, 16), (16, 64), (48, 64), (64, 64)])
def test_turned_is_a_product_of_complex_numbers(adjacent, rot, s):
    rng = np.random.default_rng(rot + s)
    x = rng.standard_normal((5, 3, s))
    angle = rng.uniform(-9, 9, (5, rot // 2))
    got = rwo.turned(x, np.concatenate([np.cos(angle), np.sin(angle)], 1), adjacent)
    for r in range(5):
        for h in range(3):
            for i in range(rot // 2):
                a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
                want = complex(x[r, h, a], x[r, h, b]) * complex(math.cos(angle[r, i]), math.sin(angle[r, i]))
                assert abs(complex(got[r, h, a], got[r, h, b]) - want) <= 1e-14 * abs(want) + 1e-300
    np.testing.assert_array_equal(got[..., rot:], x[..., rot:])


def test_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 1, 64))
    table = np.concatenate([f(np.outer(np.arange(40), 10000.0 ** (-np.arange(0, 64, 2) / 64))) for f in (np.cos, np.sin)], 1)

    def score(i, j):
        return float((rwo.turned(q, table[i:i + 1], False) * rwo.turned(k, table[j:j + 1], False)).sum())

    assert abs(score(3, 0) - score(39, 36)) < 1e-12 and abs(score(5, 5) - float((q * k).sum())) < 1e-12


@pytest.mark.parametrize("adjacent", [False, True])
def test_turned_bits(adjacent):
    rng = np.random.default_rng(3)
    bits = synth.f32_to_bf16_bits(rng.standard_normal((30, 2, 64)).astype(np.float32))
    table = rwo.angle_table(30, 32)
    got = orc.from_bf16_bits(rwo.turned_bits(bits, table, adjacent))
    x = orc.from_bf16_bits(bits)
    exact = table.astype(np.float64)
    want = rwo.turned(x, exact, adjacent)
    # |a cos| + |b sin| and |b cos| + |a sin|: the sum of one sign or the other
    size = np.maximum(*(np.abs(rwo.turned(np.abs(x), np.abs(exact) * np.repeat([1, sign], 16), adjacent)) for sign in (1, -1)))
    # two products and a sum in fp32, 2^-24 of their size each (and a little for their errors' products), and the result's rounding
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) + 4 * 2.0 ** -24 * size).all()
    np.testing.assert_array_equal(rwo.turned_bits(bits, table[:1].repeat(30, 0), adjacent), bits)     # position 0
    np.testing.assert_array_equal(rwo.turned_bits(bits, table, adjacent)[..., 32:], bits[..., 32:])


def test_seen():
    assert rwo.seen(5, 2, 0).tolist() == [3, 4]
    assert rwo.seen(5, 2, 1).tolist() == [0, 3, 4]
    assert rwo.seen(5, 1, 9).tolist() == rwo.seen(5, 5, 0).tolist() == rwo.seen(5, 99, 0).tolist() == [0, 1, 2, 3, 4]
    assert rwo.seen(0, 3, 2).tolist() == []
    for l in range(1, 12):
        for window in range(1, 13):
            for sinks in range(13):
                want = [j for j in range(l) if l - 1 - j < window or j < sinks]
                assert rwo.seen(l, window, sinks).tolist() == want


@pytest.mark.parametrize("n,n_kv,l,window,sinks", [(4, 4, 9, 3, 2), (8, 2, 33, 10, 0), (6, 1, 20, 40, 5)])
def test_attend_window_is_a_masked_softmax(n, n_kv, l, window, sinks):
    rng = np.random.default_rng(n + l)
    q, k, v = rng.standard_normal((n, 16)), rng.standard_normal((l, n_kv, 16)), rng.standard_normal((l, n_kv, 16))
    got, _, _, keys = rwo.attend_window(q, k, v, window, sinks)
    mask = torch.tensor([l - 1 - j < window or j < sinks for j in range(l)])
    assert keys == int(mask.sum())
    for h in range(n):
        kk, vv = (torch.from_numpy(x[:, h // (n // n_kv)]) for x in (k, v))
        p = torch.softmax(torch.where(mask, kk @ torch.from_numpy(q[h]) / 4, -math.inf), 0)
        np.testing.assert_allclose(got[h], (p @ vv).numpy(), rtol=1e-12, atol=1e-13)
