"""The whole-stack loop on a pool of 8 bits, layer by layer on what the layer was given and what its pages hold."""
import numpy as np
import pytest
import torch

from oracle import ds_oracle as orc
from oracle import kv_quant_oracle as kvo
from paper_2401_09670_amd import instance as inst
from paper_2401_09670_amd import synth
from tests import gpu_util as gu
from tests.kv_pages import KINDS
from tests.test_gpu_quant_steps import _check_step, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,n_kv,overlap", [("e4m3", 0, False), ("int8", 2, True)])
def test_small_stack_runs_a_workload_to_completion(gpu, kind, n_kv, overlap):
    shape = synth.ModelShape(hidden=512, n_heads=4, head_dim=128, ffn=1024, n_layers=3, n_kv_heads=n_kv)
    rng = np.random.default_rng(12)
    reqs = [inst.Request(i, int(rng.integers(1, 150)), int(rng.integers(1, 24))) for i in range(20)]
    life = [synth.blocks_needed(r.prompt_len + r.output_len - 1, 16) for r in reqs]
    pool = max(life) * 3                                   # tight: admission has to wait for pages
    stack = inst.GpuStack(shape, 3, 5, pool, max_batch=6, max_prefill_tokens=256, max_ctx=max(life) * 16,
                          max_blocks_per_seq=max(life), vocab=1024, n_pos=64, overlap_handoff=overlap, kv_cache=kind)
    stack.k_pool.fill_(0x7f)
    stack.v_pool.fill_(0x7f)
    stack.k_scale.fill_(float("nan"))
    stack.v_scale.fill_(float("nan"))
    sched = inst.Scheduler(reqs, inst.BlockPool(pool, 5), 6, 256, 16, max(life))
    stack.capture = {0: [], 2: []}
    raw = inst.run_workload(stack, sched)
    assert raw["finished"] == len(reqs) and sched.pool.n_free == pool
    assert sum(s["batch"] for s in raw["steps"]) == sum(r.output_len - 1 for r in reqs)
    for li, caps in stack.capture.items():
        w = orc.weights_from_bits(gu.host_weights(stack._keep[li]))
        steps = [c for c in caps if c["kind"] == "decode"]
        assert len(steps) == len(raw["steps"])
        for c in steps[::max(1, len(steps) // 6)]:
            pages = c["k_pool"], c["v_pool"], c["k_scale"], c["v_scale"]
            keys = [_tokens(pages, KINDS[kind], c["table"][i], int(l) + 1) for i, l in enumerate(c["ctx"])]
            _check_step(w, shape, gu.to_f64(c["x"]), c["y"], [True] * len(keys), keys, KINDS[kind])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_preloaded_contexts(gpu, kind):
    shape = synth.ModelShape(hidden=512, n_heads=4, head_dim=128, ffn=1024, n_layers=2)
    reqs = [inst.Request(i, l, 4, preloaded=True) for i, l in enumerate((40, 1, 16, 33))]
    life = [synth.blocks_needed(r.prompt_len + r.output_len - 1, 16) for r in reqs]
    stack = inst.GpuStack(shape, 2, 7, sum(life), max_batch=4, max_prefill_tokens=0, max_ctx=max(life) * 16,
                          max_blocks_per_seq=max(life), vocab=512, n_pos=64, kv_cache=kind)
    sched = inst.Scheduler(reqs, inst.BlockPool(sum(life), 5), 4, 16, 16, max(life))
    raw = inst.run_workload(stack, sched)
    assert raw["finished"] == 4 and len(raw["steps"]) == 3
    assert torch.isfinite(stack.k_scale[:, :, :, 0].float()).all()


def test_a_kind_that_there_is_not(gpu):
    with pytest.raises(ValueError, match="kv_cache"):
        inst.GpuStack(synth.TINY, 1, 1, 4, 1, 16, 16, 1, kv_cache="int4")


@pytest.mark.parametrize("kind,overlap", [("e4m3", False), ("int8", True)])
def test_handed_off_pages_are_the_oracles(gpu, kind, overlap):
    shape = synth.ModelShape(hidden=512, n_heads=4, head_dim=128, ffn=2048, n_layers=3)
    lens = [33, 16, 1, 70]
    stack = inst.GpuStack(shape, 3, 9, 40, max_batch=4, max_prefill_tokens=128, max_ctx=96, max_blocks_per_seq=6, vocab=512,
                          n_pos=128, overlap_handoff=overlap, kv_cache=kind)
    for pool, scale in ((stack.k_pool, stack.k_scale), (stack.v_pool, stack.v_scale)):
        pool.fill_(0x7f)
        scale.fill_(float("nan"))
    sched = inst.Scheduler([inst.Request(i, l, 1) for i, l in enumerate(lens)], inst.BlockPool(40, 2), 4, 128, 16, 6)
    batch = sched.next_prefill_batch()
    table = sched.prefill_table(batch)
    stack.capture = {0: [], 1: [], 2: []}
    stack.prefill(lens, [s.req.rid for s in batch], table)
    torch.cuda.synchronize()
    for li in range(3):
        cap = stack.capture[li][0]
        for rows, pool, scale, is_v in ((cap["k_out"], stack.k_pool, stack.k_scale, False),
                                        (cap["v_out"], stack.v_pool, stack.v_scale, True)):
            payload, c = kvo.quantise(gu.to_f64(rows).reshape(sum(lens), 4, -1), KINDS[kind])
            want, want_c = np.full(pool[li].shape, 0x7f, np.uint8), np.full(scale[li].shape, np.nan)
            kvo.to_pages(payload, c, lens, table, want, want_c, is_v)
            assert np.array_equal(pool[li].cpu().numpy(), want)
            assert np.array_equal(gu.to_f64(scale[li]), want_c, equal_nan=True)
