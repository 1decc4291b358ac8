"""An adapter with values that are not finite changes its own rows of
bnn_bgemm_lora and no others', on every form of its kernels."""
import pytest
import torch

import test_gpu_lora_forms as forms
from paper_1808_00209_amd import bnn

pytestmark = pytest.mark.gpu

BAD = 3  # the adapter


@pytest.mark.parametrize("algo", [bnn.ALGO_AUTO, bnn.ALGO_VALU], ids=["matrix", "vector"])
@pytest.mark.parametrize("form", forms.FORMS, ids=str)
def test_rows_of_other_adapters_keep_their_bits(form, algo):
    p = forms._inputs(form)
    order = bnn.bnn_group_rows(p["ids"], forms.ADAPTERS)[1]
    others = p["ids"] != BAD
    assert others.any() and not others.all()
    with bnn.options(algo=algo):
        want = forms._call(p)[others]
        for name in ("a", "b", "scale"):
            for value in (float("inf"), float("nan"), -float("inf")):
                bad = p[name].clone()
                if name == "scale":
                    bad[BAD] = value
                else:
                    bad[BAD, ::3, ::5] = value
                for o in (None, order):
                    got = forms._call(p, **{name: bad, "order": o})[others]
                    assert torch.equal(got, want), (name, value)


@pytest.mark.parametrize("form", forms.FORMS, ids=str)
def test_rows_without_an_adapter_are_the_binary_layer(form):
    """All adapters hold NaN: rows whose id is none give alpha S alone."""
    p = forms._inputs(form)
    none = p["ids"] < 0
    only = forms._call(p, ids=torch.full_like(p["ids"], -1))
    got = forms._call(p, a=torch.full_like(p["a"], float("nan")),
                      b=torch.full_like(p["b"], float("nan")))
    assert none.any() and torch.equal(got[none], only[none])
