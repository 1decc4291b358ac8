"""Sizes that the C side's 32-bit fields do not hold: refused by the binding, not
cut to their low bits.  CPU only: tensors without storage that say they are on
the device."""
import pytest
import torch

from paper_1808_00209_amd import bnn

FAR = 2 ** 32 + 5  # 5 in its low 32 bits


class Device(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return -1


def _t(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(Device)


i8, i32 = torch.int8, torch.int32


@pytest.mark.parametrize("call, name", [
    (lambda: bnn.bnn_logprobs(_t(1, FAR), _t(1, dtype=i32)), "V"),
    (lambda: bnn.bnn_logprobs(_t(1, 9), _t(1, FAR, dtype=i32)), "n"),
    (lambda: bnn.bnn_logprobs(_t(1, 9), top_k=FAR), "top_k"),
    (lambda: bnn.bnn_rmsnorm(_t(1, FAR)), "D"),
    (lambda: bnn.bnn_q8gemm(_t(1, FAR, dtype=i8), _t(3, FAR, dtype=i8)), "K"),
    (lambda: bnn.bnn_q8gemm(_t(1, 64, dtype=i8), _t(FAR, 64, dtype=i8)), "N"),
    (lambda: bnn.bnn_route(_t(1, FAR), 2), "E"),
    (lambda: bnn.bnn_group_rows(_t(9, dtype=i32), FAR), "G"),
    (lambda: bnn.bnn_group_rows_workspace_size(9, FAR), "G"),
    (lambda: bnn.bnn_bgemm_lora(_t(1, 64), _t(FAR, 2, dtype=i32), _t(1, dtype=i32), _t(1, 8, 64), _t(1, FAR, 8)), "N"),
    (lambda: bnn.bnn_route(_t(1, 64), 2, groups=8, top_groups=FAR), "top_groups")])
def test_refused(call, name):
    with pytest.raises(ValueError, match=name + " is -?%d: beyond 32 bits" % FAR):
        call()


@pytest.mark.parametrize("kind, sizes", [
    (bnn.RmsnormDesc, dict(M=5, D=64, dtype=0, weight_dtype=0, eps=1e-6)),
    (bnn.Q8gemmDesc, dict(M=5, N=64, K=7, dtype=0)),
    (bnn.LogprobsDesc, dict(T=5, V=64, n=1, top_k=2, dtype=0, logit_scale=1.0))])
def test_descriptions(kind, sizes):
    """By name and by place; rows are 64 bits wide, factors may be large."""
    for name, value in sizes.items():
        if isinstance(value, float):
            assert getattr(kind(**dict(sizes, **{name: 2.0 ** 90})), name) == 2.0 ** 90
            assert getattr(kind(*dict(sizes, **{name: 2.0 ** 90}).values()), name) == 2.0 ** 90
            continue
        rows = name in "MT"
        for far in ((1 << 64) + 5, -(1 << 63) - 1) if rows else (FAR, 1 << 31, -(1 << 31) - 1):
            wide = dict(sizes, **{name: far})
            with pytest.raises(ValueError, match=name):
                kind(**wide)
            with pytest.raises(ValueError, match=name):
                kind(*wide.values())
        if rows:
            assert getattr(kind(**dict(sizes, **{name: FAR})), name) == FAR
            assert getattr(kind(*dict(sizes, **{name: FAR}).values()), name) == FAR
    assert kind(**sizes).dtype == kind(*sizes.values()).dtype == 0
