"""asp_matvec on the GPU against the definition in float64 on the CPU.

Bound, element by element, derived beforehand: the one rounding of y to bf16
(2^-8 of its value), the two bf16 pieces of x~ (2^-16 of every term), and
float32 sums of at most 16384 terms (a random walk of sqrt(16384) roundings of
2^-24 is 2^-17 of the terms' sum): 2^-8 |y| * 1.01 + 2^-15 * sum |terms|.
"""

import dataclasses

import numpy as np
import pytest
import torch

from oracle import qwam_oracle as O
from paper_2609_33269_amd import qwam as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()


def _layer(K, N, r, group=64, bias=False, seed=0, smooth=True, zero_groups=False):
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(N, K, generator=g) / K ** 0.5
    if zero_groups:
        W[::3, :group] = 0.0
    lam = torch.exp(torch.randn(K, generator=g))
    b = torch.randn(N, generator=g).bfloat16().cuda() if bias else None
    if r == 0 and not smooth:
        return Q.make_plain_layer(W.cuda(), b, group=group)
    L1 = (torch.randn(K, max(r, 16), generator=g) / K ** 0.5).bfloat16()
    L2 = torch.randn(max(r, 16), N, generator=g).bfloat16()
    layer = Q.make_layer(W.cuda(), lam.cuda(), L1.cuda(), L2.cuda(), b, group=group)
    return layer if r else dataclasses.replace(layer, r=0, L1t=None, L2t=None, L1=None, L1f=None)


def _terms(layer, x):
    """y and the sum of its terms' magnitudes, float64."""
    f64 = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
    codes = O.unpack_codes(layer.wq.cpu().numpy()).astype(np.float64)
    w = codes * np.repeat(f64(layer.ws).T, layer.group, axis=1)
    xt = f64(x.float())
    if layer.inv_smooth is not None:
        xt = xt * f64(layer.inv_smooth)
    if layer.hadamard:
        xt = O.rotate_exact(xt, layer.hadamard)
    y, s = xt @ w.T, np.abs(xt) @ np.abs(w).T
    if layer.r:
        L1, L2 = f64(layer.L1t.float()).T, f64(layer.L2t.float()).T
        y, s = y + (xt @ L1) @ L2, s + (np.abs(xt) @ np.abs(L1)) @ np.abs(L2)
    if layer.bias is not None:
        b = f64(layer.bias.float())
        y, s = y + b, s + np.abs(b)
    return y, s


def _check(layer, x, y):
    ref, s = _terms(layer, x)
    err = np.abs(y.cpu().double().numpy() - ref)
    bound = 1.01 * 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * s
    assert np.isfinite(err).all() and (err <= bound).all(), f"worst {np.max(err / bound):.3f} of its bound"


def _x(M, K, seed=1):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g)
    x[:, ::37] *= 20
    return x.bfloat16().cuda()


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16])
@pytest.mark.parametrize("group", [64, 32])
def test_tokens(M, group):
    layer = _layer(1024, 272, 16, group, bias=True, seed=M)
    x = _x(M, 1024)
    _check(layer, x, Q.asp_matvec(layer, x))


@pytest.mark.parametrize("K", [64, 128, 192, 320, 576, 832, 1088, 2112, 3264, 5184, 8256, 14336, 16448])
@pytest.mark.parametrize("group", [64, 32])
def test_widths(K, group):
    for M in (1, 6):
        layer = _layer(K, 48, 32, group, seed=K)
        x = _x(M, K)
        _check(layer, x, Q.asp_matvec(layer, x))


@pytest.mark.parametrize("N", [16, 32, 48, 80, 112, 240, 1040, 4112, 9232, 20496])
def test_outputs(N):
    for M, r in ((1, 16), (5, 0), (16, 64)):
        layer = _layer(448, N, r, 64, bias=True, seed=N)
        x = _x(M, 448)
        _check(layer, x, Q.asp_matvec(layer, x))


@pytest.mark.parametrize("r", [0, 16, 32, 48, 64])
@pytest.mark.parametrize("M", [1, 3, 11])
def test_ranks(M, r):
    for K, N in ((1536, 144), (7040, 1040)):
        layer = _layer(K, N, r, 32 if r == 48 else 64, seed=r)
        x = _x(M, K)
        _check(layer, x, Q.asp_matvec(layer, x))


@pytest.mark.parametrize("M", [1, 8, 16])
@pytest.mark.parametrize("group", [64, 32])
def test_plain(M, group):
    for K, N in ((64, 16), (960, 208), (4096, 4112), (12352, 1040)):
        layer = _layer(K, N, 0, group, smooth=False, bias=N == 208, seed=K)
        x = _x(M, K)
        _check(layer, x, Q.asp_matvec(layer, x))


@pytest.mark.parametrize("group", [64, 32])
@pytest.mark.parametrize("smooth", [False, True])
def test_wide_layers(group, smooth):
    """Many output channels: wider workgroups, by the tokens' pieces; with a branch and without."""
    for r in (0, 32):
        layer = _layer(320, 16400, r, group, smooth=smooth or r > 0, seed=r)
        if not smooth:
            layer = dataclasses.replace(layer, inv_smooth=None)
        for M in (1, 3, 5, 8, 9, 16):
            x = _x(M, 320)
            _check(layer, x, Q.asp_matvec(layer, x))


@pytest.mark.parametrize("smooth", [False, True])
def test_long_rows_of_few_channels(smooth):
    """K in parts without a branch, and with one."""
    for K, N, r, group in ((16448, 48, 0, 64), (12352, 528, 0, 32), (9216, 16, 32, 64)):
        layer = _layer(K, N, r, group, smooth=smooth or r > 0, bias=N == 528)
        if not smooth:
            layer = dataclasses.replace(layer, inv_smooth=None)
        for M in (1, 2, 3, 9, 16):
            x = _x(M, K)
            _check(layer, x, Q.asp_matvec(layer, x))


@pytest.mark.parametrize("B", [16, 32, 64, 128, 256, 512, 1024])
@pytest.mark.parametrize("group", [64, 32])
def test_rotated_layers(B, group):
    """x~ rotated: its float32 butterflies (ten roundings of 2^-24 on sums of up to 1024 terms, each at most the block's
    root sum of squares) stay below the bound's 2^-15 of the terms, as every product's magnitude sum is at least a block's
    root sum of squares times that of its weights."""
    for K, N, r, M in ((1024, 272, 16, 1), (3072, 1040, 32, 5), (2048, 96, 0, 16), (5120, 144, 64, 9)):
        layer = dataclasses.replace(_layer(K, N, r, group, bias=True, seed=B), hadamard=B)
        x = _x(M, K)
        _check(layer, x, Q.asp_matvec(layer, x))
    plain = dataclasses.replace(_layer(1024, 64, 0, group, smooth=False), hadamard=B)      # without smoothing
    for M in (1, 12):
        x = _x(M, 1024)
        _check(plain, x, Q.asp_matvec(plain, x))


def test_largest_width():
    layer = _layer(65536, 32, 16, 64)
    for M in (1, 16):
        x = _x(M, 65536)
        _check(layer, x, Q.asp_matvec(layer, x))


def test_zero_scales_and_large_values():
    layer = _layer(512, 96, 16, 32, zero_groups=True)
    x = _x(4, 512)
    x[1] = 0
    x[2] *= 1e18
    x[3] *= 1e-18
    _check(layer, x, Q.asp_matvec(layer, x))


def test_calls_are_alike_and_rows_independent():
    layer = _layer(2048, 528, 32, bias=True)
    x = _x(16, 2048)
    y = Q.asp_matvec(layer, x)
    assert torch.equal(y, Q.asp_matvec(layer, x))
    out = torch.full_like(y, float("nan"))
    assert Q.asp_matvec(layer, x, out=out) is out and torch.equal(out, y)
    for M in (1, 2, 8, 13):            # a call on fewer tokens: within the same bound
        _check(layer, x[:M], Q.asp_matvec(layer, x[:M]))


def test_streams_and_graph():
    layer, x = _layer(1024, 272, 16), _x(3, 1024)
    y = Q.asp_matvec(layer, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y2 = Q.asp_matvec(layer, x, stream=s)
    s.synchronize()
    assert torch.equal(y, y2)
    xs = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = Q.asp_matvec(layer, xs)
    for i in range(4):
        xs.copy_(_x(3, 1024, seed=10 + i))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, Q.asp_matvec(layer, xs)), f"replay {i}"


@pytest.mark.parametrize("M,K,N,r,group", [(16, 4096, 528, 32, 64), (16, 1024, 272, 16, 32), (11, 8192, 80, 0, 32)])
def test_graph_of_the_larger_forms(M, K, N, r, group):
    """Workgroups with more than 64 KB of LDS, the parts' join, captured without a call before."""
    layer = _layer(K, N, r, group, smooth=r > 0)
    xs = _x(M, K)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = Q.asp_matvec(layer, xs)
    for i in range(3):
        xs.copy_(_x(M, K, seed=20 + i))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, Q.asp_matvec(layer, xs)), f"replay {i}"


def test_refusals():
    layer, x = _layer(256, 64, 16), _x(2, 256)
    with pytest.raises(Q.QwamError, match="exceeds 16"):
        Q.asp_matvec(layer, _x(17, 256))
    with pytest.raises(ValueError, match="x must have shape"):
        Q.asp_matvec(layer, _x(2, 320))
    with pytest.raises(TypeError, match="x must be torch.bfloat16"):
        Q.asp_matvec(layer, x.float())
    with pytest.raises(ValueError, match="x must be a GPU tensor"):
        Q.asp_matvec(layer, x.cpu())
    with pytest.raises(ValueError, match="x must be contiguous"):
        Q.asp_matvec(layer, _x(2, 512)[:, ::2])
    with pytest.raises(Q.QwamError, match="M must be >= 1"):
        Q.asp_matvec(layer, x[:0])
    with pytest.raises(ValueError, match="y must have shape"):
        Q.asp_matvec(layer, x, out=torch.empty(2, 48, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(Q.QwamError, match="hadamard must be"):
        Q.asp_matvec(dataclasses.replace(layer, hadamard=24), x)
    with pytest.raises(TypeError, match="L2t must be"):
        Q.asp_matvec(dataclasses.replace(layer, L2t=None), x)
    with pytest.raises(Q.QwamError, match="L1f is NULL"):
        Q.asp_matvec(dataclasses.replace(layer, L1f=None), x)
    plain = _layer(256, 64, 0, smooth=False)
    for call in (lambda: Q.asp_layer(plain, x), lambda: Q.forward(plain, x)):      # the 4-bit activation calls need the branch
        with pytest.raises(TypeError, match="inv_smooth must be"):
            call()
