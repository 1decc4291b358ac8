"""Offsets of bnn_bgemm_lora that are not finite: x + offset > 0 reads -1 where
it is NaN (as bnn_pack_bits does), and an infinite offset decides the sign."""
import numpy as np
import pytest
import torch

import test_gpu_lora_forms as forms

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", forms.FORMS, ids=str)
def test_signs_with_offsets_that_are_not_finite(form):
    M, K, _, _, kind = form
    g = np.random.default_rng(K)
    x = torch.from_numpy(g.standard_normal((M, K))).to(forms.T[kind]).cuda()
    some = np.array([np.nan, -np.nan, np.inf, -np.inf, 0.5, 3e38, -3e38], np.float32)
    some[1:2].view(np.uint32)[:] = 0xFFC00001  # a NaN with its sign set
    offset = some[g.integers(0, len(some), size=K)]
    got, want = forms._signs(form, x, offset)
    assert np.array_equal(got, want)
