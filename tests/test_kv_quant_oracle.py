"""Pins of the 8-bit cache's oracle: the formats against torch's own e4m3 and against their definition."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import synth


def _rows(seed, n=400, s=64):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, s)) * 2.0 ** rng.integers(-60, 60, (n, 1))
    return orc.from_bf16_bits(synth.f32_to_bf16_bits(x.astype(np.float32)))


def test_the_e4m3_grid_is_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(kvo.e4m3_grid(), t)


def test_e4m3_rounds_as_torch_does():
    x = _rows(1)
    b, c = kvo.quantise(x, kvo.E4M3)
    want = torch.from_numpy((x / c[:, None]).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(b, want)


@pytest.mark.parametrize("kind,top", [(kvo.E4M3, 448.0), (kvo.INT8, 127.0)])
def test_scales_are_the_least(kind, top):
    x = np.concatenate([_rows(2), np.full((1, 64), 448.0), np.full((1, 64), 450.0), np.full((1, 64), 254.0)])
    _, c = kvo.quantise(x, kind)
    a = np.abs(x).max(1)
    assert (a <= top * c).all()
    bits = synth.f32_to_bf16_bits(c.astype(np.float32))
    assert (synth.bf16_bits_to_f32(bits) == c).all()
    below = c / 2 if kind == kvo.E4M3 else synth.bf16_bits_to_f32(bits - np.uint16(1)).astype(np.float64)
    assert (a > top * below).all()


@pytest.mark.parametrize("kind", [kvo.E4M3, kvo.INT8])
def test_values_are_nearest(kind):
    x = _rows(3, 50)
    b, c = kvo.quantise(x, kind)
    grid = kvo.e4m3_grid() if kind == kvo.E4M3 else np.arange(-127, 128.0)
    grid = np.unique(grid[np.isfinite(grid)])
    v = kvo.stands_for(b, np.ones_like(c), kind)
    nearest = np.abs(x[..., None] / c[:, None, None] - grid).min(-1)
    np.testing.assert_array_equal(np.abs(x / c[:, None] - v), nearest)


@pytest.mark.parametrize("kind", [kvo.E4M3, kvo.INT8])
def test_edges(kind):
    x = np.zeros((5, 64))
    x[1, 3], x[2, 5], x[3, :] = np.nan, -np.inf, 2.0 ** -120
    x[4, 0] = 3.0
    b, c = kvo.quantise(x, kind)
    assert c[0] == 1.0 and np.isnan(c[1]) and np.isnan(c[2]) and c[3] == 2.0 ** -100 and not b[:4].any()
    assert np.isnan(kvo.stands_for(b, c, kind)[1:3]).all()


def test_ties_go_to_even():
    x = np.zeros((1, 64))
    x[0, :6] = [127.0, 0.5, 1.5, 2.5, -0.5, -1.5]
    assert list(kvo.quantise(x, kvo.INT8)[0][0, :6].view(np.int8)) == [127, 0, 2, 2, 0, -2]
    x[0, :4] = [448.0, 17.0, 19.0, -17.0]                           # steps of 2 from 16 on
    v = kvo.stands_for(*kvo.quantise(x, kvo.E4M3), kvo.E4M3)
    assert list(v[0, :4]) == [448.0, 16.0, 20.0, -16.0]


def test_attention_over_two_parts_is_that_over_both():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((8, 64)), rng.standard_normal((40, 2, 64)), rng.standard_normal((40, 2, 64))
    o, pav, _ = kvo.attend(q, k, v)
    want = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q)[:, None], torch.from_numpy(np.repeat(k, 4, 1)).permute(1, 0, 2),
        torch.from_numpy(np.repeat(v, 4, 1)).permute(1, 0, 2))[:, 0].numpy()
    np.testing.assert_allclose(o, want, rtol=1e-12, atol=1e-12)
    assert (pav >= np.abs(o) - 1e-12).all()
