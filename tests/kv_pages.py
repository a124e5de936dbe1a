"""Pages for the tests of the 8-bit cache and of shared prefixes: made by the oracle, poisoned wherever no token is."""
import numpy as np
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu

KINDS = {"bf16": binding.KV_BF16, "e4m3": binding.KV_E4M3, "int8": binding.KV_INT8}


def rows(rng, t, n_kv, s, spread=1.0):
    """bf16 rows as bits: features of unlike size, some rows far larger or smaller than the rest."""
    x = rng.standard_normal((t, n_kv, s)) * np.exp(0.4 * rng.standard_normal((n_kv, s))) * spread
    x = x * np.where(rng.random((t, n_kv, 1)) < 0.1, 2.0 ** rng.integers(-9, 4, (t, n_kv, 1)), 1.0)
    return synth.f32_to_bf16_bits(x.astype(np.float32))


class Cache:
    """A cache of `kind` that holds `lens` tokens of sequences with room for `room` (default: lens)."""

    def __init__(self, kind, lens, n_kv, s, seed, room=None, spread=1.0, k_bits=None, v_bits=None):
        rng = np.random.default_rng(seed)
        self.kind, self.name, self.n_kv, self.s, self.lens = KINDS[kind], kind, n_kv, s, [int(l) for l in lens]
        t = sum(self.lens)
        self.k_bits = rows(rng, t, n_kv, s, spread) if k_bits is None else k_bits
        self.v_bits = rows(rng, t, n_kv, s, spread) if v_bits is None else v_bits
        self.table, self.nb = synth.make_block_tables([max(1, int(c)) for c in (room or self.lens)], 16, seed)
        k, v = orc.from_bf16_bits(self.k_bits), orc.from_bf16_bits(self.v_bits)
        if self.kind == binding.KV_BF16:
            # NaN bit patterns where no token is
            kp = np.full((self.nb, n_kv, 16, s), 0x7fc1, np.uint16)
            vp = kp.copy()
            r = 0
            for i, n in enumerate(self.lens):
                for j in range(n):
                    kp[self.table[i][j // 16], :, j % 16] = self.k_bits[r]
                    vp[self.table[i][j // 16], :, j % 16] = self.v_bits[r]
                    r += 1
            self.k, self.v = gu.to_dev(kp), gu.to_dev(vp)
            self.ks = self.vs = None
            self.k_rows, self.v_rows = k, v
            return
        # 0x7f: NaN as e4m3; NaN scales
        kp, vp = np.full((self.nb, n_kv, 16, s), 0x7f, np.uint8), np.full((self.nb, n_kv, s, 16), 0x7f, np.uint8)
        ks, vs = np.full((self.nb, n_kv, 16), np.nan), np.full((self.nb, n_kv, 16), np.nan)
        kb, kc = kvo.quantise(k, self.kind)
        vb, vc = kvo.quantise(v, self.kind)
        kvo.to_pages(kb, kc, self.lens, self.table, kp, ks, False)
        kvo.to_pages(vb, vc, self.lens, self.table, vp, vs, True)
        self.host = dict(k=kp, v=vp, ks=ks, vs=vs)
        self.k, self.v = torch.from_numpy(kp).cuda(), torch.from_numpy(vp).cuda()
        self.ks, self.vs = scales_dev(ks), scales_dev(vs)
        self.k_rows, self.v_rows = kvo.stands_for(kb, kc, self.kind), kvo.stands_for(vb, vc, self.kind)

    def seq(self, i):
        """K and V of sequence i as the cache holds them."""
        a = sum(self.lens[:i])
        return self.k_rows[a:a + self.lens[i]], self.v_rows[a:a + self.lens[i]]

    @property
    def args(self):
        return self.k, self.v, self.ks, self.vs, self.nb, self.kind


def scales_dev(c: np.ndarray) -> torch.Tensor:
    bits = synth.f32_to_bf16_bits(np.where(np.isnan(c), 1.0, c).astype(np.float32))
    assert (synth.bf16_bits_to_f32(bits) == np.where(np.isnan(c), 1.0, c)).all(), "a scale is a bf16"
    return gu.to_dev(np.where(np.isnan(c), np.uint16(0x7fc0), bits))


def scales_host(t: torch.Tensor) -> np.ndarray:
    return t.float().cpu().numpy().astype(np.float64)


def close(got, o, p_abs_v, size, s, keys):
    """Entries of `got` that are further from `o` than the bound (both [.., n, s])."""
    bound = kvo.attention_bound(o, p_abs_v, size, s, keys)
    bad = ~(np.abs(got - o) <= bound)
    return [] if not bad.any() else [(tuple(i), got[tuple(i)], o[tuple(i)], bound[tuple(i)]) for i in np.argwhere(bad)[:4]]
