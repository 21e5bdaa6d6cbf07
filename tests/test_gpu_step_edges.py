"""Edges of a single token's step on the GPU."""

import dataclasses

import numpy as np
import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import block
from paper_2609_33269_amd import qwam as Q
from test_gpu_block_norm import _backward_check, _inputs
from test_gpu_matvec import _layer, _terms, _x
from test_gpu_paged_attention import _cache, _check, _q

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


# ---- block_norm under autograd ----

@pytest.mark.parametrize("post", [False, True])
def test_unread_parameters_without_a_branch(post):
    """The norm in front of the first block reads neither gate nor post_weight: they get no gradient, the others theirs."""
    p, dh, _ = _inputs(6, 72, 2)
    if not post:
        p["post_weight"] = None
    leaf = {n: t.clone().requires_grad_() for n, t in p.items() if t is not None and n != "branch"}
    kw = {n: leaf.get(n) for n in ("gate", "post_weight", "weight", "scale", "shift")}
    _, h = P.block_norm(leaf["x"], post_norm=post, **kw)
    h.backward(dh)
    want = P.block_norm_backward(None, dh, p["x"], post_norm=post, **{n: p[n] for n in kw})
    for n, t in leaf.items():
        if n in ("gate", "post_weight"):
            assert t.grad is None, n
        else:
            assert torch.equal(t.grad, want["d" + n].to(torch.bfloat16)), n


@pytest.mark.parametrize("used", ["x", "h"])
def test_unused_outputs_have_no_gradient_tensor(used, monkeypatch):
    """A last block uses one output only: the other's gradient is taken as none, not as a tensor of zeros."""
    p, dh, dxo = _inputs(10, 72, 2)
    d = dxo.bfloat16().cuda()
    kw = {n: p[n] for n in ("gate", "weight", "scale", "shift")}
    x, b = (p[n].clone().requires_grad_() for n in ("x", "branch"))
    seen = []
    call = block.block_norm_backward
    monkeypatch.setattr(block, "block_norm_backward", lambda *a, **k: seen.append(a[0]) or call(*a, **k))
    xo, h = P.block_norm(x, b, residual_scale=0.5, **kw)
    if used == "x":
        xo.backward(d)
        assert torch.equal(x.grad, (0.5 * d.float()).bfloat16())
        assert torch.equal(b.grad, (d.float() * kw["gate"].float().repeat_interleave(5, 0)).bfloat16())
    else:
        h.backward(dh)
        assert seen == [None]
        want = call(None, dh, xo.detach(), p["branch"], residual_scale=0.5, **kw)
        assert torch.equal(x.grad, want["dx"]) and torch.equal(b.grad, want["dbranch"])


# ---- operators without a gradient ----

def _tracked_calls():
    """(call, tensors of it that a gradient could be asked of), fresh tensors."""
    layer = _layer(256, 64, 16, bias=True)
    x = _x(2, 256)
    yield "asp_matvec", lambda: P.asp_matvec(layer, x), [x, layer.L2t, layer.L1f, layer.bias, layer.ws, layer.inv_smooth]
    yield "asp_matvec", lambda: P.asp_matvec(layer, x, stream=torch.cuda.current_stream()), [x]
    for fp8 in (False, True):
        cache = _cache([30, 40], 2, 64, 16, fp8=fp8)
        q, L = _q(2, 4, 64), torch.tensor([30, 40], dtype=torch.int32, device="cuda")
        held = [cache.k_scale, cache.v_scale] if fp8 else [cache.k, cache.v]
        yield "paged_attention", lambda: P.paged_attention(cache, q, L), [q] + held
        k, v = _q(2, 2, 64, 3), _q(2, 2, 64, 4)
        seq = torch.arange(2, dtype=torch.int32, device="cuda")
        yield "kv_append", lambda: P.kv_append(cache, k, v, seq, L), [k, v] + held


def test_no_gradient_vanishes():
    """They have none: an input that requires one is refused, and taken where no gradient is recorded."""
    for name, call, tensors in _tracked_calls():
        for t in tensors:
            call()
            t.requires_grad_()
            with pytest.raises(ValueError, match=f"requires a gradient, which {name} does not have"):
                call()
            with torch.no_grad():
                call()
            t.requires_grad_(False)


def test_no_tangent_vanishes():
    import torch.autograd.forward_ad as fwd
    layer, x = _layer(256, 64, 16), _x(2, 256)
    cache = _cache([30, 40], 2, 64, 16)
    q, k, L = _q(2, 4, 64), _q(2, 2, 64, 3), torch.tensor([30, 40], dtype=torch.int32, device="cuda")
    with fwd.dual_level():
        dual = lambda t: fwd.make_dual(t, torch.ones_like(t))  # noqa: E731
        for name, call in (("asp_matvec", lambda: P.asp_matvec(layer, dual(x))),
                           ("paged_attention", lambda: P.paged_attention(cache, dual(q), L)),
                           ("kv_append", lambda: P.kv_append(cache, dual(k), k, L * 0, L)),
                           ("kv_append", lambda: P.kv_append(cache, k, dual(k), L * 0, L))):
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(ValueError, match=f"carries a tangent, which {name} does not"):
                    call()
        P.asp_matvec(layer, x)


def test_block_norm_refuses_tangents():
    """It has a gradient but no forward-mode derivative."""
    import torch.autograd.forward_ad as fwd
    p, dh, _ = _inputs(6, 72, 2)
    with fwd.dual_level():
        for name in p:
            kw = {n: (fwd.make_dual(t, torch.ones_like(t)) if n == name else t) for n, t in p.items()}
            x, b = kw.pop("x"), kw.pop("branch")
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(ValueError, match=f"{name} carries a tangent, which block_norm does not"):
                    P.block_norm(x, b, post_norm=True, **kw)
            with pytest.raises(ValueError, match=f"{'x_out' if name == 'x' else name} carries a tangent, which block_norm_backward"):
                P.block_norm_backward(None, dh, x, b, post_norm=True, **kw)


# ---- infinities ----

@pytest.mark.parametrize("group", [64, 32])
@pytest.mark.parametrize("smooth", [False, True])
@pytest.mark.parametrize("K,N", [(320, 272), (12352, 48)])
def test_matvec_of_infinities(K, N, smooth, group):
    """An infinite or NaN channel gives what the definition gives, in that token alone: infinities of their sign, NaN
    where its code is 0 or two of them meet."""
    layer = _layer(K, N, 0, group, smooth=smooth, bias=True)
    inf = float("inf")
    for M in (1, 2, 4, 7, 8, 16):
        x = _x(M, K)
        finite = P.asp_matvec(layer, x)
        for bad in ([(17, inf)], [(0, -inf), (K - 1, -inf)], [(40, inf), (41, -inf)], [(3, float("nan"))]):
            m = (M - 1) // 2
            y = x.clone()
            for k, v in bad:
                y[m, k] = v
            with np.errstate(invalid="ignore"):
                want = torch.from_numpy(_terms(layer, y[m:m + 1])[0][0])
            got = P.asp_matvec(layer, y)
            assert torch.equal(got[m].double().cpu().nan_to_num(nan=7.0), want.nan_to_num(nan=7.0)), f"{M} tokens, {bad}"
            others = [i for i in range(M) if i != m]
            assert torch.equal(got[others], finite[others])


def test_rotated_matvec_of_infinities():
    """A rotation spreads one over its block: the token is NaN, the others are what they were."""
    layer = dataclasses.replace(_layer(512, 64, 16), hadamard=64)
    x = _x(5, 512)
    want = P.asp_matvec(layer, x)
    x[3, 100] = float("inf")
    got = P.asp_matvec(layer, x)
    assert got[3].isnan().all() and torch.equal(got[[0, 1, 2, 4]], want[[0, 1, 2, 4]])


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("length", [40, 700, 5000])
def test_attention_of_infinite_scores(length, D):
    """Scores of -inf have weight 0; where all of them are, the result is zeros; one of +inf makes it NaN, as a softmax."""
    cache = _cache([length] * 2, 2, D, 64)
    q = _q(2, 6, D).abs() + 0.125
    L = torch.full((2,), length, dtype=torch.int32, device="cuda")
    want = P.paged_attention(cache, q, L)
    row = lambda b, p: (int(cache.table[b, p // 64]), slice(None), p % 64)  # noqa: E731
    gone = list(range(0, length, 3))
    for p in gone:
        cache.k[row(0, p)] = -float("inf")
    got = P.paged_attention(cache, q, L)
    assert torch.equal(got[1], want[1]) and torch.isfinite(got).all()
    # the same as without these positions
    keep = [p for p in range(length) if p % 3]
    packed = _cache([len(keep)], 2, D, 64)
    for i, p in enumerate(keep):
        for c, o in ((packed.k, cache.k), (packed.v, cache.v)):
            c[int(packed.table[0, i // 64]), :, i % 64] = o[row(0, p)]
    _check(packed, q[:1], [len(keep)], got[:1])
    cache.k[row(1, length // 2)] = float("inf")
    got = P.paged_attention(cache, q, L)
    assert got[1].isnan().all() and torch.isfinite(got[0]).all()
    for p in range(length):
        cache.k[row(0, p)] = -float("inf")
    assert (P.paged_attention(cache, q, L)[0] == 0).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("length", [40, 5000])
def test_attention_of_values_that_are_not_finite(length, fp8):
    """They reach their channel of their heads' results only, where these are not finite."""
    cache = _cache([length] * 2, 2, 128, 64, fp8=fp8)
    q, L = _q(2, 6, 128), torch.full((2,), length, dtype=torch.int32, device="cuda")
    want = P.paged_attention(cache, q, L)
    for bad in (float("nan"),) if fp8 else (float("nan"), float("inf"), -float("inf")):
        v = cache.v.clone().view(torch.uint8 if fp8 else torch.bfloat16)
        v[int(cache.table[1, 0]), 1, 5, 77] = 0x7F if fp8 else bad
        got = P.paged_attention(P.PagedCache(cache.k, v.view(cache.v.dtype), cache.table, cache.k_scale, cache.v_scale), q, L)
        assert not torch.isfinite(got[1, 3:, 77]).any()
        got[1, 3:, 77] = want[1, 3:, 77]
        assert torch.equal(got, want)


# ---- a table wider than the contexts ----

@pytest.mark.parametrize("fp8", [False, True])
def test_graph_over_a_wide_table(fp8):
    """A program records its step with a table for the longest context it will allow, and replays it from the first
    token on: the ranges are laid out for the table, the sequences fill few of them."""
    H, D, page, width = 2, 128, 64, 1024
    lengths = [0, 1, 100, 700, 9000, 5]
    cache = _cache([n + 1 for n in lengths], H, D, page, fp8=fp8, width=width)
    q = _q(len(lengths), 3 * H, D)
    L = torch.zeros(len(lengths), dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = P.paged_attention(cache, q, L)
    for now in ([0] * 6, [min(n, 1) for n in lengths], lengths, [n // 2 for n in lengths], [lengths[4 - i] if i < 5 else 5 for i in range(6)]):
        now = [min(n, m + 1) for n, m in zip(now, lengths)]
        L.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.paged_attention(cache, q, L)), f"lengths {now}"
        _check(cache, q, now, out)
