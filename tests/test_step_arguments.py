"""Arguments of a wrong kind in a token's step are named, on the host too."""

import os

import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import qwam as Q


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(Q.LIB_PATH):
        from paper_2609_33269_amd import build
        build.build()


X = torch.zeros(4, 64, dtype=torch.bfloat16)


@pytest.mark.parametrize("name", ["gate", "scale", "shift"])
@pytest.mark.parametrize("value", [[1.0], 0.5, "0"])
def test_norm_parameters_that_are_no_tensors(name, value):
    for grad in (True, False):
        with torch.set_grad_enabled(grad), pytest.raises(TypeError, match=f"{name} must be a torch.Tensor"):
            P.block_norm(X, X, **{name: value})
        with torch.set_grad_enabled(grad), pytest.raises(TypeError, match=f"{name} must be a torch.Tensor"):
            P.block_norm_backward(X, X, X, X, **{name: value})


@pytest.mark.parametrize("name", ["weight", "post_weight"])
def test_norm_weights_that_are_no_tensors(name):
    for grad in (True, False):
        with torch.set_grad_enabled(grad), pytest.raises(TypeError, match=f"{name} must be a torch.Tensor"):
            P.block_norm(X, X, post_norm=True, **{name: [1.0]})


@pytest.mark.parametrize("value", [None, 1.0, [[1.0]], torch.zeros(4), torch.zeros(2, 2, 64)])
def test_norm_rows(value):
    with pytest.raises(ValueError, match="x must be a tensor of two dimensions"):
        P.block_norm(value, X)
    with pytest.raises(ValueError, match="x_out must be a tensor of two dimensions"):
        P.block_norm_backward(X, X, value, X)
