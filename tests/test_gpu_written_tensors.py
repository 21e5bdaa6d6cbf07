"""Tensors that a caller gives to be written are seen by autograd as changed: what an earlier operation saved of them no
longer enters its gradient silently.  Every call is made natively and, with a stream, through ctypes."""

import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import qwam as Q
from test_gpu_matvec import _layer, _x
from test_gpu_paged_attention import _cache, _q

pytestmark = pytest.mark.gpu

FP4 = torch.float4_e2m1fn_x2
STREAM = [False, True]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rope():
    plan, pos, x = P.rope_plan((16, 16)), _int([[1, 2], [3, 4], [5, 6]]), _q(3, 4, 32)
    other = torch.empty_like(x)
    yield "rope in place", lambda **kw: P.rope(x, pos, plan, out=x, **kw), [x]
    yield "rope", lambda **kw: P.rope(x, pos, plan, out=other, **kw), [other]


def _caches():
    at = _int([0, 1, 1]), _int([3, 5, 6])
    k, v = _q(3, 2, 64), _q(3, 2, 64, 2)
    for name in ("bf16", "fp8", "fp4"):
        if name == "fp4":
            c = P.new_cache(8, 2, 64, 2, 4, 16, FP4)
            c.table[:] = torch.arange(8, dtype=torch.int32).view(2, 4)
        else:
            c = _cache([30, 40], 2, 64, 16, fp8=name == "fp8")
        written = [c.k, c.v] + ([c.k_scale, c.v_scale] if name == "fp4" else [])
        yield "kv_append " + name, lambda c=c, **kw: P.kv_append(c, k, v, *at, **kw), written
        out = torch.empty_like(k), torch.empty_like(v)
        yield "kv_read " + name, lambda c=c, out=out, **kw: P.kv_read(c, *at, out=out, **kw), list(out)
        o, q = torch.empty(2, 6, 64, dtype=torch.bfloat16, device="cuda"), _q(2, 6, 64)
        yield "paged_attention " + name, lambda c=c, o=o, q=q, **kw: P.paged_attention(c, q, _int([10, 12]), out=o, **kw), [o]


def _layers():
    layer, x = _layer(256, 64, 16, bias=True), _x(4, 256)
    acts = [(torch.empty(4, 128, dtype=torch.uint8, device="cuda"), torch.empty(4, 4, device="cuda"),
             torch.empty(4, 16, dtype=torch.bfloat16, device="cuda")) for _ in range(3)]
    ys = [torch.empty(4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    yield "quantize_act", lambda **kw: P.quantize_act(layer, x, out=acts[0], **kw), list(acts[0])
    yield "quantize_act_deflated", lambda **kw: P.quantize_act_deflated(layer, x, out=acts[1], **kw), list(acts[1])
    given = P.quantize_act(layer, x)
    yield "asp_linear", lambda **kw: P.asp_linear(layer, *given, out=ys[0], **kw), [ys[0]]
    yield "asp_layer", lambda **kw: P.asp_layer(layer, x, out=ys[1], **kw), [ys[1]]
    yield "asp_layer with its activations", lambda **kw: P.asp_layer(layer, x, out=ys[2], act_out=acts[2], **kw), [ys[2], *acts[2]]
    yield "asp_matvec", lambda **kw: P.asp_matvec(layer, x, out=ys[3], **kw), [ys[3]]
    b, h = _x(4, 256, 2), torch.empty_like(x)
    s = x.clone()
    yield "block_norm in place", lambda **kw: P.block_norm(s, b, out=(s, h), **kw), [s, h]
    h2 = torch.empty_like(x)
    yield "block_norm without a branch", lambda **kw: P.block_norm(x, out=(None, h2), **kw), [h2]
    A = torch.zeros(256, 256, device="cuda")
    yield "aog_accumulate", lambda **kw: P.aog_accumulate(_x(256, 64), A, **kw), [A]


@pytest.mark.parametrize("stream", STREAM)
@pytest.mark.parametrize("calls", [_rope, _caches, _layers])
def test_versions(calls, stream):
    for name, call, written in calls():
        before = [t._version for t in written]
        call(**({"stream": torch.cuda.current_stream()} if stream else {}))
        assert all(t._version > n for t, n in zip(written, before)), name


@pytest.mark.parametrize("stream", STREAM)
def test_what_is_read_keeps_its_version(stream):
    kw = {"stream": torch.cuda.current_stream()} if stream else {}
    plan, pos, x, c = P.rope_plan((16, 16)), _int([[1, 2], [3, 4], [5, 6]]), _q(3, 4, 32), _cache([30, 40], 2, 64, 16)
    k = _q(3, 2, 64)
    at = _int([0, 1, 1]), _int([3, 5, 6])
    layer, y = _layer(256, 64, 16), _x(4, 256)
    read = [x, pos, plan.inv_freq, k, *at, c.table, y, layer.ws, layer.L1f]
    before = [t._version for t in read]
    P.rope(x, pos, plan, **kw)
    P.kv_append(c, k, k, *at, **kw)
    cache = [c.k._version, c.v._version]
    P.kv_read(c, *at, **kw)
    P.paged_attention(c, _q(2, 6, 64), _int([10, 12]), **kw)
    P.asp_matvec(layer, y, **kw)
    P.block_norm(y, y, **kw)
    assert before == [t._version for t in read] and cache == [c.k._version, c.v._version]


@pytest.mark.parametrize("stream", STREAM)
def test_saved_tensors_that_were_written(stream):
    """An operation with a learned factor saved x; a view of x, or x, is then overwritten: its backward pass raises."""
    kw = {"stream": torch.cuda.current_stream()} if stream else {}
    plan, pos = P.rope_plan((16, 16)), _int([[1, 2], [3, 4], [5, 6]])
    for view in (False, True):
        wide = _q(3, 6, 32)
        x = wide[:, 1:5] if view else wide
        w = torch.ones((), dtype=torch.bfloat16, device="cuda", requires_grad=True)
        z = (wide * w).sum()
        P.rope(x, pos, plan, out=x, **kw)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()
    c = _cache([30, 40], 2, 64, 16)
    z = (c.k.nan_to_num() * w).sum() + (c.v * w).sum()
    P.kv_append(c, _q(3, 2, 64), _q(3, 2, 64), _int([0, 1, 1]), _int([3, 5, 6]), **kw)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()


@pytest.mark.parametrize("stream", STREAM)
def test_tensors_of_inference_mode(stream):
    """They have no version; the calls write them as before, within the mode and outside."""
    kw = {"stream": torch.cuda.current_stream()} if stream else {}
    with torch.inference_mode():
        plan, pos, x = P.rope_plan((16, 16)), _int([[1, 2], [3, 4], [5, 6]]), _q(3, 4, 32)
        c, k = _cache([30, 40], 2, 64, 16), _q(3, 2, 64)
        at = _int([0, 1, 1]), _int([3, 5, 6])
        want = P.rope(x, pos, plan, **kw)
        P.kv_append(c, k, k, *at, **kw)
        a, b = P.kv_read(c, *at, **kw)
        assert torch.equal(a, k) and torch.equal(b, k)
    P.kv_append(c, k, k, *at, **kw)
    assert P.rope(x, pos, plan, out=x, **kw) is x
    with torch.inference_mode():
        assert torch.equal(x, want)


@pytest.mark.parametrize("stream", STREAM)
def test_outputs_that_require_a_gradient(stream):
    """They are refused where autograd records: what is written has no history."""
    kw = {"stream": torch.cuda.current_stream()} if stream else {}
    c, q = _cache([30, 40], 2, 64, 16), _q(2, 6, 64)
    layer, x = _layer(256, 64, 16), _x(4, 256)
    o, y, h = torch.empty_like(q), torch.empty(4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    for t, name, call in ((o, "out requires a gradient, which paged_attention", lambda: P.paged_attention(c, q, _int([10, 12]), out=o, **kw)),
                          (y, "out requires a gradient, which asp_matvec", lambda: P.asp_matvec(layer, x, out=y, **kw)),
                          (h, "block_norm under autograd takes neither out", lambda: P.block_norm(x, x, out=(x.clone(), h), **kw))):
        t.requires_grad_()
        with pytest.raises(ValueError, match=name):
            call()
        with torch.no_grad():
            call()
