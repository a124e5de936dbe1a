"""The debug validation of ds_decode_step_shared: the page that a row's new token goes to is no prefix's and no other row's.
Every bad call is refused on the host, before anything is launched."""
import pytest
import torch

from paper_2401_09670_amd import binding, synth
from tests import gpu_util as gu
from tests.kv_pages import KINDS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "int8"])
def test_a_new_page_has_one_owner(gpu, kind):
    shape, nb, kind = synth.TINY, 12, KINDS[kind]
    ctx, h, n, s = gu.make_ctx(shape), shape.hidden, shape.kv_heads, shape.head_dim
    ctx.ds_set_validate(True)
    lw, _keep = gu.weights_to_dev(synth.make_layer_weights(shape, 1))
    quant = kind != binding.KV_BF16
    k, v = (torch.zeros(nb, n, 16, s, dtype=torch.uint8 if quant else torch.bfloat16, device="cuda") for _ in range(2))
    ks, vs = (torch.ones(nb, n, 16, dtype=torch.bfloat16, device="cuda") if quant else None for _ in range(2))
    x, y = (torch.zeros(3, h, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = gu.workspace(ctx.ds_decode_shared_workspace_bytes(3, 32, 48))

    def step(bt, lens=(17, 0, -1), pt=((0, 1), (2, 3)), prefix=(32, 9), cug=(0, 2, 3)):
        ctx.ds_decode_step_shared(lw, x, gu.i32_dev(cug), 2, 2, gu.i32_dev(prefix), gu.i32_dev(pt), 2, 32, gu.i32_dev(lens),
                                  gu.i32_dev(bt), 3, 3, 48, k, v, ks, vs, nb, kind, y, ws)
        torch.cuda.synchronize()

    good = [[4, 5, -1], [6, -1, -1], [-1, -1, -1]]
    step(good)
    # a page that a prefix names but that none of its tokens needs, and one that is in a table of a row behind its end
    step([[4, 3, -1], [6, 5, -1], [-1, -1, -1]])
    # the first of two own pages of rows may be one: none of them is written
    step([[4, 5, -1], [4, 6, -1], [4, -1, -1]], lens=(17, 20, -1))

    def refused(text, bt, **kw):
        before = [t.clone() for t in (k, v, ks, vs) if t is not None]
        with pytest.raises(binding.DsError) as e:
            step(bt, **kw)
        assert e.value.status == 5 and text in str(e.value), str(e.value)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(before, (t for t in (k, v, ks, vs) if t is not None)))

    refused("row 1 writes into block 1, which is prefix 0's", [[4, 5, -1], [1, -1, -1], [-1, -1, -1]])
    refused("row 0 writes into block 2, which is prefix 1's", [[4, 2, -1], [6, -1, -1], [-1, -1, -1]])   # another group's
    refused("row 1 writes into block 0, which is prefix 0's", [[4, 5, -1], [0, -1, -1], [-1, -1, -1]])
    refused("row 1 writes into block 4, which is row 0's", [[4, 5, -1], [4, -1, -1], [-1, -1, -1]])      # its earlier page
    refused("row 0 writes into block 7, which is row 2's", [[4, 7, -1], [6, -1, -1], [8, 7, 9]], lens=(17, 0, 40))
    # the same new page twice: on 8 bits named by the check of the appends
    refused("block 6", [[4, 6, -1], [6, -1, -1], [-1, -1, -1]])


def test_a_prefix_that_no_row_has_counts(gpu):
    """Its pages hold tokens that a later step attends over."""
    shape = synth.TINY
    ctx, h, n, s = gu.make_ctx(shape), shape.hidden, shape.kv_heads, shape.head_dim
    ctx.ds_set_validate(True)
    lw, _keep = gu.weights_to_dev(synth.make_layer_weights(shape, 1))
    k, v = (torch.zeros(6, n, 16, s, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x, y = (torch.zeros(1, h, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = gu.workspace(ctx.ds_decode_shared_workspace_bytes(1, 16, 16))

    def step(page):
        ctx.ds_decode_step_shared(lw, x, gu.i32_dev([0, 0, 1]), 2, 1, gu.i32_dev([16, 3]), gu.i32_dev([[0], [1]]), 1, 16,
                                  gu.i32_dev([2]), gu.i32_dev([[page]]), 1, 1, 16, k, v, None, None, 6, 0, y, ws)

    step(2)
    with pytest.raises(binding.DsError) as e:
        step(0)
    assert e.value.status == 5 and "prefix 0's" in str(e.value)
