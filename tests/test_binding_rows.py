"""What the binding tells the library of a tensor's rows: their true distance,
and a refusal where rows overlap (a broadcast row, sliding windows), whose
elements are fewer than rows times row length.  CPU only: a host tensor that
says it is on the device is looked at and never read."""
import pytest
import torch

from paper_1808_00209_amd import bnn


class Device(torch.Tensor):
    """A host tensor that passes for one on the device."""
    is_cuda = True


def _on_device(t):
    return t.as_subclass(Device)


@pytest.mark.parametrize("rows, cols, stride", [(4, 8, 8), (4, 8, 11), (1, 8, 8), (0, 8, 8),
                                                (5, 1, 1), (5, 1, 7), (4, 3, 4)])
def test_the_distance_of_rows(rows, cols, stride):
    t = torch.zeros(64).as_strided((rows, cols), (stride, 1))
    want = stride if rows > 1 else cols
    assert bnn._rows(_on_device(t), "x") == want


def test_one_row_of_any_stride():
    for stride in (0, 3, 100):
        t = torch.zeros(300).as_strided((1, 8), (stride, 1))
        assert bnn._rows(_on_device(t), "x") == 8


@pytest.mark.parametrize("overlapping", [
    torch.zeros(1, 64).expand(4096, 64), torch.zeros(64).expand(3, 64),
    torch.zeros(320).unfold(0, 64, 8), torch.zeros(10).as_strided((3, 4), (3, 1)),
    torch.zeros(1, 1).expand(5, 1)], ids=lambda t: "%s by %s" % (tuple(t.shape), t.stride()))
def test_overlapping_rows_are_refused(overlapping):
    x = _on_device(overlapping)
    with pytest.raises(ValueError, match="overlap"):
        bnn._rows(x, "x")
    with pytest.raises(ValueError, match="overlap"):
        bnn.bnn_route(x, 1)
    n, k = 8, x.shape[1]
    with pytest.raises(ValueError, match="overlap"):
        bnn.bnn_bgemm_lora(x, _on_device(torch.zeros((n, bnn.words(k)), dtype=torch.int32)),
                           _on_device(torch.zeros(x.shape[0], dtype=torch.int32)),
                           _on_device(torch.zeros(1, 8, k)), _on_device(torch.zeros(1, n, 8)))


@pytest.mark.parametrize("shape", [(), (8,), (8, 64), (1, 8, 63), (1, 1, 8, 64)], ids=str)
def test_adapters_of_another_shape_are_refused(shape):
    x = _on_device(torch.zeros(4, 64))
    with pytest.raises(ValueError, match="a must have shape"):
        bnn.bnn_bgemm_lora(x, _on_device(torch.zeros((8, 2), dtype=torch.int32)),
                           _on_device(torch.zeros(4, dtype=torch.int32)),
                           _on_device(torch.zeros(shape)), _on_device(torch.zeros(1, 8, 8)))
