"""Edges of a single token's step on the GPU."""

import pytest
import torch

from paper_2609_33269_amd import qwam as Q
from test_gpu_block_norm import _backward_check, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()


# ---- block_norm_backward without eps ----

@pytest.mark.parametrize("D", [64, 520, 1001, 2048, 4096])
@pytest.mark.parametrize("T,S", [(1, 1), (3, 1), (10, 2), (21, 3)])
def test_backward_without_eps(T, S, D):
    """Rows that do not fill a workgroup's last turn: what stands in for the missing ones has no deviation to divide by."""
    for norm, post, f32 in (("rms", True, False), ("rms", False, True), ("layer", True, True), ("layer", False, False)):
        p, dh, dxo = _inputs(T, D, S, f32, seed=D + T)
        _backward_check(p, dh, dxo, norm, post, eps=0.0)
