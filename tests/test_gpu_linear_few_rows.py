"""Products of nine to 64 rows in groups of eight (FP32, and BF16 weights off the 16-byte grid), and what lies beside them."""
import pytest
import torch

import layer_model as lm
import test_gpu_linear as tl

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_b200 as t
    return t


# Up to T I O of 2^24 (FP32) and 2^23 (BF16), and where eight rows of x fit the shared memory, they go by groups; beyond, to the tensor cores.
@pytest.mark.parametrize("dt,pitched", [(F32, False), (F32, True), (BF, False), (BF, True)])
@pytest.mark.parametrize("T", [9, 15, 16, 33, 63, 64, 65])
@pytest.mark.parametrize("I,O", [(7, 33), (77, 91), (250, 100), (511, 250), (511, 257), (700, 375), (1023, 512), (3070, 41), (3075, 41)])
def test_groups_of_rows(tsr, T, I, O, dt, pitched):
    tl.check_forward(tsr, T, I, O, dt=dt, kind="silu", p=0.2, residual=True, pitched=pitched)


@pytest.mark.parametrize("kind", lm.ACTS)
def test_groups_of_rows_and_the_same_rows_alone(tsr, kind):
    """A group's rows are computed as they are in a call of their own, but for the words of dropout, which go by the row of the call."""
    x, w, b = tl.make((21, 301), F32, 1), tl.make((70, 301), F32, 2, 0.1), tl.make((1, 70), F32, 3)[0]
    y, _ = tsr.linear_forward(x, w, b, activation=kind)
    for at in (0, 8):
        one, _ = tsr.linear_forward(x[at:at + 8], w, b, activation=kind)
        assert torch.equal(one, y[at:at + 8])
    d = tsr.Dropout(0.5, 3, 4)
    z, _ = tsr.linear_forward(x, w, b, activation=kind, dropout=d)
    assert torch.equal(z, tsr.dropout_forward(y, d))
