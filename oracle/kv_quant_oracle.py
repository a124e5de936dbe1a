"""CPU oracle for the 8-bit paged cache and for attention behind a shared prefix.  TEST INFRASTRUCTURE.

Numpy, in 64 bits, from the formats' definition (``include/ds.h``); independent of the kernels, which it is compared with.
A row is the last axis: the ``s`` numbers of one token and key/value head.
"""
from __future__ import annotations

import numpy as np

E4M3, INT8 = 1, 2
PAGE = 16


def e4m3_grid() -> np.ndarray:
    """The value of each of the 256 bytes: sign, 4 exponent bits (bias 7), 3 mantissa bits; S.1111.111 is NaN."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(b & 128, -v, v)


def bf16_up(x: np.ndarray) -> np.ndarray:
    """The least bf16 >= x (x > 0, in bf16's normal range)."""
    step = 2.0 ** (np.floor(np.log2(x)) - 7)
    return np.ceil(x / step) * step


def quantise(x: np.ndarray, kind: int):
    """x [..., s] (bf16 numbers) -> (bytes uint8 [..., s], scales float64 [...])."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x).all(-1)
    a = np.where(fine, np.abs(np.where(np.isfinite(x), x, 0.0)).max(-1), 0.0)
    some = np.where(a > 0, a, 1.0)
    if kind == E4M3:
        e = np.ceil(np.log2(some / 448.0))
        e = np.where(some > 448.0 * 2.0 ** e, e + 1, e)          # (the logarithm's last place)
        e = np.where(some <= 448.0 * 2.0 ** (e - 1), e - 1, e)
        c = 2.0 ** np.maximum(e, -100.0)
    else:
        c = np.maximum(bf16_up(some / 127.0), 2.0 ** -100)
    c = np.where(a > 0, c, 1.0)
    v = np.where(fine[..., None], np.where(np.isfinite(x), x, 0.0) / c[..., None], 0.0)
    if kind == E4M3:
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6))) - 3)
        v = np.rint(v / step) * step                             # (rint: ties to even)
        grid = np.abs(e4m3_grid()[:127])
        b = np.searchsorted(grid, np.abs(v)).astype(np.uint8)
        assert (grid[b] == np.abs(v)).all()
        # a negative number that rounds to nothing is minus zero
        b = b | np.where(np.signbit(np.where(fine[..., None], x, 0.0)), np.uint8(128), np.uint8(0))
    else:
        b = np.rint(v).astype(np.int8).view(np.uint8)
    return b, np.where(fine, c, np.nan)


def stands_for(b: np.ndarray, c: np.ndarray, kind: int) -> np.ndarray:
    """What bytes [..., s] and scales [...] stand for, exactly."""
    v = e4m3_grid()[b] if kind == E4M3 else b.view(np.int8).astype(np.float64)
    return v * np.asarray(c, np.float64)[..., None]


def to_pages(rows_b: np.ndarray, rows_c: np.ndarray, lens, table, pages: np.ndarray, scales: np.ndarray, is_v: bool):
    """Packed rows [t, n_kv, s] and scales [t, n_kv] into pages ([nb, n_kv, 16, s], V: [nb, n_kv, s, 16]), in place."""
    r = 0
    for i, n in enumerate(lens):
        for j in range(int(n)):
            p, s = int(table[i][j // PAGE]), j % PAGE
            if is_v:
                pages[p, :, :, s] = rows_b[r]
            else:
                pages[p, :, s] = rows_b[r]
            scales[p, :, s] = rows_c[r]
            r += 1


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray):
    """One query [n, s] over [L, n_kv, s]: (output [n, s], sum_j p_j |v_j| [n, s], largest sum_d |q_d k_d| / sqrt(s) [n])."""
    n, s = q.shape
    if k.shape[0] == 0:
        return np.zeros((n, s)), np.zeros((n, s)), np.zeros(n)
    g = n // k.shape[1]
    kk, vv = np.repeat(k, g, 1), np.repeat(v, g, 1)
    z = np.einsum("hd,lhd->hl", q, kk) / np.sqrt(s)
    size = (np.einsum("hd,lhd->hl", np.abs(q), np.abs(kk)) / np.sqrt(s)).max(1)
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    return np.einsum("hl,lhd->hd", p, vv), np.einsum("hl,lhd->hd", p, np.abs(vv)), size


def attention_bound(o: np.ndarray, p_abs_v: np.ndarray, size: np.ndarray, s: int, keys: int) -> np.ndarray:
    """How far a kernel may be from `o` that sums in fp32 and rounds the probabilities and the result to bf16.

    The result: 2^-8 of it.  A probability times its scale, rounded: 2^-8 of it, so 2^-8 sum p |v|.  A score is a sum of s
    products in fp32: off by at most (s + 3) 2^-24 sum |q_d k_d| / sqrt(s) (with the scale's and the factor's own
    roundings), the same for the maximum; what is exponentiated is rounded once more, to 2^-24 of at most that size.  A
    probability then changes by that much of itself, in the numerator and in the sum.  Sums over `keys` terms and the
    merging of states: (keys + 64) 2^-24."""
    score = 2 * ((s + 3) * 2.0 ** -24 + 2.0 ** -23) * size
    rest = 2 * score + (keys + 64) * 2.0 ** -23
    return 2.0 ** -8 * np.abs(o) * 1.01 + (2.0 ** -8 + rest[..., None]) * p_abs_v * 1.01 + 1e-30
