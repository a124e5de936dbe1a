"""CPU oracle for positions by rotation and for attention through a sliding window.  TEST INFRASTRUCTURE.

Numpy, from the definitions of ``include/ds.h``; independent of the kernels, which it is compared with.
"""
from __future__ import annotations

import numpy as np

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo


def angle_table(n_pos: int, rot: int, base: float = 10000.0) -> np.ndarray:
    """[n_pos, rot] float32: rot / 2 cosines, then rot / 2 sines of position times base^(-2 i / rot)."""
    angle = np.arange(n_pos)[:, None] * base ** (-np.arange(0, rot, 2) / rot)
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)


def _pairs(x: np.ndarray, rot: int, adjacent: bool):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if adjacent else (x[..., :rot // 2], x[..., rot // 2:rot])


def turned(x: np.ndarray, rows: np.ndarray, adjacent: bool) -> np.ndarray:
    """x [t, heads, s] by the table's rows [t, rot], in the type that both are given in: in float32 each product and each sum is
    rounded by itself, as the definition says; in float64 the value that this approximates."""
    rot = rows.shape[1]
    a, b = _pairs(x, rot, adjacent)
    cos, sin = rows[:, None, :rot // 2], rows[:, None, rot // 2:]
    out = x.copy()
    to_a, to_b = _pairs(out, rot, adjacent)                # (views)
    with np.errstate(invalid="ignore", over="ignore"):
        to_a[...], to_b[...] = a * cos - b * sin, b * cos + a * sin
    return out


def turned_bits(bits: np.ndarray, rows: np.ndarray, adjacent: bool) -> np.ndarray:
    """bf16 bits [t, heads, s] -> the bits of the turned rows; features from rot on as they are."""
    from paper_2401_09670_amd import synth
    rot = rows.shape[1]
    x = orc.from_bf16_bits(bits).astype(np.float32)
    out = synth.f32_to_bf16_bits(turned(x, rows.astype(np.float32), adjacent))
    out[..., rot:] = bits[..., rot:]
    return out


def seen(length: int, window: int, sinks: int) -> np.ndarray:
    """The tokens that the last of `length` sees: j with length - 1 - j < window or j < sinks."""
    j = np.arange(length)
    return j[(length - 1 - j < window) | (j < sinks)]


def attend_window(q: np.ndarray, k: np.ndarray, v: np.ndarray, window: int, sinks: int):
    """kv_quant_oracle.attend of one query [n, s] over what it sees of the tokens [L, n_kv, s], and how many those are."""
    at = seen(len(k), window, sinks)
    return kvo.attend(q, k[at], v[at]) + (len(at),)
