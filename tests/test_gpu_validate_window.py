"""The debug validation of attention through a window takes the batches that the call does, empty sequences among them."""
import pytest

from paper_2401_09670_amd import binding
from tests import gpu_util as gu
from tests.test_gpu_prefill_window import Call, _ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[20, 0, 13], [0, 5], [7, 0, 0], [0, 0, 1]], ids=str)
def test_empty_sequences(gpu, lens):
    n, s = 4, 64
    ctx = _ctx(n, n, s)
    ctx.ds_set_validate(True)
    Call(n, n, s, lens, 4).run(ctx, 5, 1).check(5, 1)


@pytest.mark.parametrize("cu", [[0, 20, 19, 33], [0, 0, 34, 33], [1, 20, 20, 33], [0, 0, 0, 33], [0, 20, 33, 34]], ids=str)
def test_batches_that_are_none(gpu, cu):
    """Lengths below 0 and above the bound, a beginning that is not 0, an end behind the rows."""
    n, s = 4, 64
    ctx = _ctx(n, n, s)
    ctx.ds_set_validate(True)
    c = Call(n, n, s, [20, 0, 13], 4)
    c.cu = gu.i32_dev(cu)
    with pytest.raises(binding.DsError) as e:
        c.run(ctx, 5, 1)
    assert e.value.status == 5
    assert (c.o == 9.0).all()
