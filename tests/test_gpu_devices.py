"""Every call runs on the current device, and refuses tensors and streams of another."""

import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import qwam as Q
from test_gpu_matvec import _layer, _x
from test_gpu_paged_attention import _cache, _q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()


def _calls():
    layer, x = _layer(256, 64, 16, bias=True), _x(4, 256)
    acts = P.quantize_act(layer, x)
    yield "quantize_act", lambda **kw: P.quantize_act(layer, x, **kw)
    yield "quantize_act_deflated", lambda **kw: P.quantize_act_deflated(layer, x, **kw)
    yield "asp_linear", lambda **kw: P.asp_linear(layer, *acts, **kw)
    yield "asp_layer", lambda **kw: P.asp_layer(layer, x, **kw)
    yield "asp_matvec", lambda **kw: P.asp_matvec(layer, x, **kw)
    yield "debug_group_partials", lambda **kw: P.debug_group_partials(layer, acts[0], **kw)
    g, one = torch.randn(64, 256, device="cuda"), torch.ones(256, device="cuda")
    yield "pack_weights", lambda **kw: P.pack_weights(g, one, **kw)
    A = torch.zeros(256, 256, device="cuda")
    yield "aog_accumulate", lambda **kw: P.aog_accumulate(_x(256, 64), A, **kw)
    B = torch.eye(256, device="cuda")
    yield "aog_protected_basis", lambda **kw: P.aog_protected_basis(B, 16, **kw)
    gate = _x(1, 256, 3)
    yield "block_norm", lambda **kw: P.block_norm(x, x, gate=gate, **kw)
    yield "block_norm_backward", lambda **kw: P.block_norm_backward(x, x, x, x, gate=gate, **kw)
    c, q, n = _cache([30, 40], 2, 64, 16), _q(2, 2, 64), torch.tensor([10, 12], dtype=torch.int32, device="cuda")
    yield "kv_append", lambda **kw: P.kv_append(c, q, q, n * 0, n, **kw)
    yield "kv_read", lambda **kw: P.kv_read(c, n * 0, n, **kw)
    yield "paged_attention", lambda **kw: P.paged_attention(c, q, n, **kw)
    plan = P.rope_plan((64,))
    yield "rope", lambda **kw: P.rope(q, n[:, None], plan, **kw)


def test_tensors_of_another_device(monkeypatch):
    """(One device is enough: with the current one said to be another, its tensors are of another device.  Calls with a stream
    check their arguments in Python.)"""
    s = torch.cuda.current_stream()
    for name, call in _calls():
        call()
        call(stream=s)
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "current_device", lambda: 1)
            m.setattr(Q._native(), "quantize", lambda *a: None)
            with pytest.raises(ValueError, match=f"is on cuda:0, {name} runs on the current device cuda:1"):
                call(stream=s)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="two GPUs")
def test_two_devices():
    for name, call in _calls():
        with torch.cuda.device(1), pytest.raises(ValueError, match=f"is on cuda:0, {name} runs on the current device cuda:1"):
            call()
