"""New rows of Q, K and V turned by their positions and appended to a paged cache: every bit against the oracle's."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from oracle import rotary_window_oracle as rwo
from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu
from tests.kv_pages import KINDS, rows, scales_dev

pytestmark = pytest.mark.gpu

SHAPES = [(4, 4, 64), (8, 2, 128), (5, 5, 128), (16, 1, 128), (64, 8, 128), (12, 3, 64)]
N_POS = 700


def _ctx(n, n_kv, s):
    return binding.Context(n * s, n, s, 64, n_kv_heads=n_kv)


class Call:
    """A call's data: rows of a QKV product (with `pad` elements behind each), poisoned pages, and the outputs."""

    def __init__(self, n, n_kv, s, kind, new, before, rot, adjacent, seed, one=False, positions=None, pad=0, extra=0,
                 table=None):
        rng = np.random.default_rng(seed)
        self.n, self.n_kv, self.s, self.kind, self.name = n, n_kv, s, KINDS[kind], kind
        self.new, self.before, self.adjacent, self.rot = list(new), list(before), adjacent, rot
        self.t = sum(new) + extra
        self.q_bits, self.k_bits, self.v_bits = (rows(rng, self.t, h, s) for h in (n, n_kv, n_kv))
        self.stride = (n + 2 * n_kv) * s + pad
        qkv = np.full((self.t, self.stride), 0x7fc1, np.uint16)
        qkv[:, :self.stride - pad] = np.concatenate([self.q_bits, self.k_bits, self.v_bits], 1).reshape(self.t, -1)
        self.qkv = gu.to_dev(qkv)
        flat = self.qkv.view(-1)
        self.q, self.k, self.v = flat, flat[n * s:], flat[(n + n_kv) * s:]
        self.table = rwo.angle_table(N_POS, rot) if table is None else table
        self.positions = positions
        room = [max(0, b) + r + 17 for b, r in zip(before, new)]
        self.tables, self.nb = synth.make_block_tables(room, 16, seed + 1)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        if kind == "bf16":
            kc, vc = (torch.randint(-2 ** 15, 2 ** 15, (self.nb, n_kv, 16, s), dtype=torch.int16, device="cuda",
                                    generator=g).view(torch.bfloat16) for _ in range(2))
            self.pages = (kc, vc, None, None)
        else:
            kc = torch.randint(0, 256, (self.nb, n_kv, 16, s), dtype=torch.uint8, device="cuda", generator=g)
            vc = torch.randint(0, 256, (self.nb, n_kv, s, 16), dtype=torch.uint8, device="cuda", generator=g)
            sc = torch.randint(-2 ** 15, 2 ** 15, (2, self.nb, n_kv, 16), dtype=torch.int16, device="cuda", generator=g)
            self.pages = (kc, vc, sc[0].view(torch.bfloat16), sc[1].view(torch.bfloat16))
        self.was = [None if x is None else x.clone() for x in self.pages]
        self.cu_np = synth.cu_seqlens(new)
        self.cu = None if one else gu.i32_dev(self.cu_np)
        self.q_out = torch.full((self.t, n, s), 7.0, dtype=torch.bfloat16, device="cuda")
        self.k_out = torch.full((self.t, n_kv, s), 7.0, dtype=torch.bfloat16, device="cuda")
        self.table_dev, self.bt, self.lens = torch.from_numpy(self.table).cuda(), gu.i32_dev(self.tables), gu.i32_dev(before)
        self.pos_dev = None if positions is None else gu.i32_dev(positions)

    def run(self, ctx, k_out=True):
        ctx.ds_kv_append_rotary(self.q, self.stride, self.k, self.v, self.stride, self.cu, len(self.new), self.t, self.lens,
                                self.pos_dev, self.table_dev, len(self.table), self.rot, self.adjacent, self.bt,
                                self.tables.shape[1], *self.pages, self.nb, self.kind, self.q_out,
                                self.k_out if k_out else None)
        return self

    def check(self, k_out=True):
        torch.cuda.synchronize()
        seven = np.full(1, 0x40e0, np.uint16)[0]
        pos, there = np.zeros(self.t, int), np.zeros(self.t, bool)
        for i, (b, r) in enumerate(zip(self.before, self.new)):
            if b >= 0:
                a = self.cu_np[i]
                pos[a:a + r], there[a:a + r] = b + np.arange(r), True
        turn = np.clip(pos if self.positions is None else np.asarray(self.positions), 0, len(self.table) - 1)
        q, k = (rwo.turned_bits(x, self.table[turn], self.adjacent) for x in (self.q_bits, self.k_bits))
        want_q, want_k = np.where(there[:, None, None], q, seven), np.where(there[:, None, None], k, seven)
        np.testing.assert_array_equal(gu.to_bits(self.q_out), want_q)
        np.testing.assert_array_equal(gu.to_bits(self.k_out), want_k if k_out else np.full_like(want_k, seven))
        to = [None if x is None else (x.cpu().numpy().copy() if x.dtype == torch.uint8 else gu.to_bits(x).copy())
              for x in self.was]
        if self.kind:
            (kb, kc), (vb, vc) = (kvo.quantise(orc.from_bf16_bits(x), self.kind) for x in (k, self.v_bits))
            kc, vc = gu.to_bits(scales_dev(kc)), gu.to_bits(scales_dev(vc))
        for i, (b, r) in enumerate(zip(self.before, self.new)):
            for j in range(r if b >= 0 else 0):
                p, slot, row = self.tables[i][(b + j) // 16], (b + j) % 16, self.cu_np[i] + j
                if self.kind:
                    to[0][p, :, slot], to[1][p, :, :, slot], to[2][p, :, slot], to[3][p, :, slot] = kb[row], vb[row], kc[row], vc[row]
                else:
                    to[0][p, :, slot], to[1][p, :, slot] = k[row], self.v_bits[row]
        for name, got, want in zip(("k", "v", "k_scale", "v_scale"), self.pages, to):
            if got is None:
                continue
            got = got.cpu().numpy() if got.dtype == torch.uint8 else gu.to_bits(got)
            bad = np.argwhere(got != want)
            assert not len(bad), (name, len(bad), bad[0], got[tuple(bad[0])], want[tuple(bad[0])])


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s", SHAPES)
def test_one_row_of_each_sequence(gpu, n, n_kv, s, kind):
    """Single tokens, at the first slot of a page, its last, and between; one sequence pads the batch."""
    ctx = _ctx(n, n_kv, s)
    for seed, before in enumerate(([0], [15, 16, 31], [5, -1, 600, 47, 0])):
        for rot, adjacent in ((s, False), (s // 2, True), (16, False), (48, False), (48, True)):
            Call(n, n_kv, s, kind, [1] * len(before), before, rot, adjacent, seed, one=True, pad=8 * seed).run(ctx).check()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("n,n_kv,s", SHAPES)
def test_prompts_and_pieces(gpu, n, n_kv, s, kind):
    """Rows of several sequences from the first token on and from the middle of a page, some with none, one that pads the batch;
    rows behind the last sequence are left out."""
    ctx = _ctx(n, n_kv, s)
    cases = (([1], [0]), ([16], [0]), ([17, 3, 32, 1], [0] * 4), ([40, 0, 2, 33, 5], [3, 8, 15, 17, 46]),
             ([0, 7, 20, 0, 14], [0, 1, -1, 5, 2]), ([100, 1, 31], [31, 600, 16]))
    for seed, (new, before) in enumerate(cases):
        rot, adjacent = ((s, False), (s // 2, True), (32, False), (s, True), (16, True), (48, False))[seed]
        for extra in (0, 5):
            Call(n, n_kv, s, kind, new, before, rot, adjacent, seed, pad=8 * (seed % 3), extra=extra).run(ctx).check()
        Call(n, n_kv, s, kind, new, before, rot, adjacent, seed + 9).run(ctx, k_out=False).check(k_out=False)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
def test_many_rows_and_sequences(gpu, kind):
    """Several heads a wave, and more sequences than a wave looks through at once."""
    n, n_kv, s = 40, 40, 128
    Call(n, n_kv, s, kind, [700, 300], [0, 9], s, False, 3, table=rwo.angle_table(1200, s)).run(_ctx(n, n_kv, s)).check()
    n, n_kv, s = 8, 2, 64
    rng = np.random.default_rng(5)
    new, before = rng.integers(0, 9, 150), rng.integers(-1, 60, 150)
    Call(n, n_kv, s, kind, new, before, 32, True, 4).run(_ctx(n, n_kv, s)).check()
    Call(n, n_kv, s, kind, [1] * 150, before, 64, False, 5, one=True).run(_ctx(n, n_kv, s)).check()


@pytest.mark.parametrize("adjacent", [False, True])
def test_positions_of_their_own(gpu, adjacent):
    """Rows' positions given, those outside the table as the nearest in it."""
    n, n_kv, s = 8, 2, 128
    new, before = [5, 12], [0, 30]
    positions = np.array([3, 0, N_POS - 1, N_POS, 2 ** 31 - 1, -1, -2 ** 31] + list(range(40, 50)))
    for kind in ("bf16", "int8"):
        Call(n, n_kv, s, kind, new, before, s, adjacent, 6, positions=positions).run(_ctx(n, n_kv, s)).check()


@pytest.mark.parametrize("adjacent", [False, True])
def test_near_the_value_in_64_bits(gpu, adjacent):
    """Against the rotation in 64 bits by the same table: two products and a sum, each rounded to fp32 (2^-24 of itself, so
    2^-24 (|a cos| + |b sin|) for the products together and that again for the sum), then to bf16 (2^-8)."""
    n, n_kv, s = 8, 8, 64
    c = Call(n, n_kv, s, "bf16", [60], [0], s, adjacent, 8).run(_ctx(n, n_kv, s))
    torch.cuda.synchronize()
    for got, bits in ((c.q_out, c.q_bits), (c.k_out, c.k_bits)):
        x, rows_ = orc.from_bf16_bits(bits), c.table[:60].astype(np.float64)
        want = rwo.turned(x, rows_, adjacent)
        size = np.abs(rwo.turned(np.abs(x), np.abs(rows_) * np.repeat([1.0, -1.0], s // 2), adjacent))  # |a cos| + |b sin|, and
        size = np.maximum(size, np.abs(rwo.turned(np.abs(x), np.abs(rows_), adjacent)))                  # |b cos| + |a sin|
        assert (np.abs(gu.to_f64(got) - want) <= 2.0 ** -8 * np.abs(want) + 2.02 * 2.0 ** -24 * (1 + 2.0 ** -8) * size).all()


def test_infinities_and_nan_stay_in_their_pairs(gpu):
    """A number that is not finite reaches the two of its pair, and in 8 bits its row."""
    n, n_kv, s = 4, 2, 64
    for kind in ("bf16", "e4m3"):
        c = Call(n, n_kv, s, kind, [3], [2], 32, False, 12)
        bits = np.concatenate([c.q_bits, c.k_bits, c.v_bits], 1)
        bits[0, 1, 3], bits[1, n, 20], bits[2, n + 1, 50], bits[1, n + 2, 0] = 0x7f80, 0xff80, 0x7fc0, 0x7f80
        c.q_bits, c.k_bits, c.v_bits = bits[:, :n], bits[:, n:n + n_kv], bits[:, n + n_kv:]
        c.qkv.copy_(gu.to_dev(bits.reshape(3, -1)))
        c.run(_ctx(n, n_kv, s))
        torch.cuda.synchronize()
        for got, x in ((c.q_out, c.q_bits), (c.k_out, c.k_bits)):
            want = orc.from_bf16_bits(rwo.turned_bits(x, c.table[2:5], False))
            np.testing.assert_array_equal(gu.to_f64(got), want)
            assert np.isnan(want).sum() + np.isinf(want).sum() > 0
        if kind == "e4m3":
            sc = gu.to_f64(c.pages[2])
            page, slots = c.tables[0][0], np.arange(2, 5)
            assert np.isnan(sc[page, 0, 3]) and np.isnan(sc[page, 1, 4]) and np.isfinite(sc[page, 0, 2])
            assert np.isnan(gu.to_f64(c.pages[3])[page, 0, 3])


def test_in_place(gpu):
    """q_out = q and k_out = k, where rows follow each other."""
    n, n_kv, s = 16, 4, 128
    ctx = _ctx(n, n_kv, s)
    for one in (False, True):
        c = Call(n, n_kv, s, "bf16", [1] * 9 if one else [50, 3], [4] * 9 if one else [0, 18], s, False, 13, one=one)
        q, k = gu.to_dev(c.q_bits), gu.to_dev(c.k_bits)
        c.q_out, c.k_out = q, k
        ctx.ds_kv_append_rotary(q, n * s, k, gu.to_dev(c.v_bits), n_kv * s, c.cu, len(c.new), c.t, c.lens, None, c.table_dev,
                                len(c.table), s, 0, c.bt, c.tables.shape[1], *c.pages, c.nb, c.kind, q, k)
        c.check()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_captured_and_replayed(gpu, kind):
    """One row of each sequence in a graph, whose inputs change between the replays; on a stream of its own."""
    n, n_kv, s = 8, 2, 128
    ctx = _ctx(n, n_kv, s)
    c = Call(n, n_kv, s, kind, [1] * 5, [3, 16, 31, 200, -1], s, False, 14, one=True)
    c.run(ctx)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.run(ctx)
    for step in range(3):
        other = Call(n, n_kv, s, kind, [1] * 5, [4 + step, 40, -1, 201, step], s, False, 20 + step, one=True)
        c.qkv.copy_(other.qkv)
        c.lens.copy_(other.lens)
        c.q_out.fill_(7.0)
        c.k_out.fill_(7.0)
        for p, w in zip(c.pages, c.was):
            if p is not None:
                p.copy_(w)
        graph.replay()
        c.q_bits, c.k_bits, c.v_bits, c.before = other.q_bits, other.k_bits, other.v_bits, other.before
        c.check()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("one", [False, True])
def test_rows_and_pages_behind_4_gib(gpu, kind, one):
    """Rows and pages that lie further behind their start than 32 bits reach."""
    n, n_kv, s = 8, 2, 128
    new, before = ([1] * 40, list(range(5, 45))) if one else ([30, 0, 11], [7, 3, 0])
    ctx = _ctx(n, n_kv, s)
    near, c = (Call(n, n_kv, s, kind, new, before, s, False, 30, one=one) for _ in range(2))
    near.run(ctx).check()
    c.stride = 1 << 26                                         # 40 rows are 5 GiB
    flat = torch.empty(c.t * c.stride, dtype=torch.bfloat16, device="cuda")
    flat.view(c.t, c.stride)[:, :c.qkv.shape[1]] = c.qkv
    c.q, c.k, c.v = flat, flat[n * s:], flat[(n + n_kv) * s:]
    far = (5 << 30) // c.pages[0][0].nbytes

    def behind(x):
        big = torch.empty((far + c.nb,) + tuple(x.shape[1:]), dtype=x.dtype, device="cuda")
        big[far:] = x
        return big

    c.pages = tuple(None if x is None else behind(x) for x in c.pages)
    c.bt = gu.i32_dev(np.where(c.tables < 0, -1, c.tables + far))
    c.nb += far
    c.run(ctx)
    torch.cuda.synchronize()
    assert torch.equal(c.q_out, near.q_out) and torch.equal(c.k_out, near.k_out)
    for x, y in zip(c.pages, near.pages):
        assert x is None or torch.equal(x[far:].view(torch.uint8), y.view(torch.uint8))


def test_validation(gpu):
    n, n_kv, s = 4, 2, 64
    ctx = _ctx(n, n_kv, s)
    ctx.ds_set_validate(True)

    def call(**change):
        c = Call(n, n_kv, s, "e4m3", [20, 3], [5, 0], 32, False, 15)
        for k, v in change.items():
            setattr(c, k, v)
        c.run(ctx)
        return c

    call().check()
    bt = call().tables
    wrong = [dict(cu=gu.i32_dev([1, 20, 23])), dict(cu=gu.i32_dev([0, 24, 23])), dict(cu=gu.i32_dev([0, 20, 24])),
             dict(lens=gu.i32_dev([5, -2])), dict(lens=gu.i32_dev([16 * bt.shape[1] - 19, 0])), dict(lens=gu.i32_dev([690, 0])),
             dict(pos_dev=gu.i32_dev([0] * 22 + [N_POS])), dict(pos_dev=gu.i32_dev([-1] * 23)),
             dict(bt=gu.i32_dev(np.where(bt == bt[0, 1], -1, bt))), dict(bt=gu.i32_dev(np.where(bt == bt[1, 0], bt[0, 1], bt)))]
    for change in wrong:
        with pytest.raises(binding.DsError) as e:
            call(**change)
        assert e.value.status == 5, change
    # pages that nothing is written to need not be there, rows of a padding sequence may have any position
    c = Call(n, n_kv, s, "e4m3", [3, 4], [33, -1], 32, False, 16, positions=[1, 2, 3, -5, -5, -5, -5])
    c.bt = gu.i32_dev(np.where(np.arange(c.tables.shape[1]) < 2, -1, c.tables))
    c.run(ctx).check()
