"""Rotary positions on the GPU against float64.

Bound of an output, derived beforehand: one rounding (bf16 2^-8 of the value, float32 2^-24), and of |x_a| + |x_b| the
errors of cos and sin (2^-22), of the two products and their sum in float32 (2^-23), and of the angle (2^-50 of it)."""

import types

import numpy as np
import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import qwam as Q

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()


def _reference(x, pos, plan, inverse=False):
    """y in float64 and the magnitudes that its bound goes by: |x_a| + |x_b| and the angle of each channel."""
    x = x.detach().cpu().double().numpy()
    T, H, D = x.shape
    f, axis = plan.inv_freq.cpu().double().numpy(), plan.axis.cpu().numpy()
    p = pos.cpu().double().numpy()[np.arange(T) % len(pos)]
    n = len(f)
    known = (axis >= 0) & (axis < p.shape[1])
    angle = np.where(known, p[:, np.where(known, axis, 0)] * f, 0.0)[:, None]
    c, s = np.cos(angle), np.sin(angle) * (-1 if inverse else 1)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if plan.interleaved else (slice(0, n), slice(n, 2 * n))
    y, mag, far = x.copy(), np.zeros_like(x), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    mag[..., a] = mag[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    far[..., a] = far[..., b] = np.abs(angle)
    return y, mag, far


def _check(x, pos, plan, got, inverse=False):
    y, mag, far = _reference(x, pos, plan, inverse)
    e = np.abs(got.detach().cpu().double().numpy() - y)
    step = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    bound = 1.001 * step * np.abs(y) + mag * (2.0 ** -22 + 2.0 ** -23 + 2.0 ** -50 * far)
    worst = float((e / np.maximum(bound, 1e-300)).max())
    assert got.dtype == x.dtype
    assert worst <= 1, f"worst {worst:.3f} of its bound"
    rest = slice(2 * len(plan.inv_freq), None)
    assert torch.equal(got[..., rest], x[..., rest])


def _x(T, H, D, f32=False, seed=0):
    x = torch.randn(T, H, D, generator=torch.Generator().manual_seed(seed))
    return (x if f32 else x.bfloat16()).cuda()


def _pos(n, axes, f32=False, seed=1, far=5000):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(-far, far, (n, axes), generator=g)
    return (p * 0.37 if f32 else p.int()).cuda()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("D,dims", [(64, (64,)), (128, (44, 42, 42)), (128, (32, 48, 48)), (96, (48, 48)), (80, (20, 22, 22)), (72, (72,)), (2, (2,)),
                                    (3, (2,)), (7, (4, 2)), (6, (6,)), (12, (4, 4, 4)), (128, (16,)), (256, (64, 64, 64, 64)), (100, (50, 50)),
                                    (34, (16, 16)), (512, (512,)), (1000, (998,))])
def test_widths(D, dims, f32, interleaved):
    plan = P.rope_plan(dims, interleaved=interleaved)
    for T, H in ((1, 1), (5, 3), (33, 20)):
        x, pos = _x(T, H, D, f32, D), _pos(T, len(dims), f32)
        for inverse in (False, True):
            _check(x, pos, plan, P.rope(x, pos, plan, inverse=inverse), inverse)


@pytest.mark.parametrize("T,S,H", [(1, 1, 48), (4, 1, 20), (7, 7, 5), (1000, 4, 2), (4096, 2, 3), (333, 3, 33), (20000, 1, 1), (2, 1, 500)])
def test_tokens_and_heads(T, S, H):
    """Few tokens of many heads, many of one, samples that share their positions."""
    for interleaved in (False, True):
        plan = P.rope_plan((44, 42, 42), interleaved=interleaved)
        x, pos = _x(T, H, 128, seed=T), _pos(T // S, 3)
        _check(x, pos, plan, P.rope(x, pos, plan))


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    """Up to the ends of int32, and as far in float32: whole turns drop out exactly."""
    plan = P.rope_plan((64, 64), interleaved=interleaved)
    ends = torch.tensor([[2 ** 31 - 1, -2 ** 31], [2 ** 30 + 1, 123456789], [0, 1], [-1, 2 ** 24 + 1]], dtype=torch.int32).cuda()
    x = _x(4, 3, 128, True)
    _check(x, ends, plan, P.rope(x, ends, plan))
    far = torch.tensor([[1e9, -3e9], [2.0 ** 40, 0.1], [1e-30, -0.0], [123456.789, 0.5]]).cuda()
    _check(x, far, plan, P.rope(x, far, plan))
    # frequencies of another kind: zero, large, whole turns
    odd = P.RopePlan(torch.tensor([0.0, 1e6, -3.0, 6.2831855, 1e-8, 1.5707964, 0.78539819, 3.1415927]).cuda(), torch.zeros(8, dtype=torch.int32).cuda(), interleaved)
    x, pos = _x(40, 2, 16, True), torch.arange(40, dtype=torch.int32)[:, None].cuda()
    _check(x, pos, odd, P.rope(x, pos, odd))


def test_axes_that_do_not_exist():
    """Their pairs do not turn, whatever the positions hold."""
    for interleaved in (False, True):
        plan = P.rope_plan((16, 16), interleaved=interleaved)
        plan.axis[3], plan.axis[9], plan.axis[15] = 2, -1, 2 ** 31 - 1
        for D in (32, 33):
            x, pos = _x(10, 3, D), _pos(10, 2)
            y = P.rope(x, pos, plan)
            _check(x, pos, plan, y)
            for i in (3, 9, 15):
                at = slice(2 * i, 2 * i + 2) if interleaved else slice(i, i + 17, 16)
                assert torch.equal(y[..., at], x[..., at])


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T", [5, 300])
def test_pairs_without_an_axis_are_copied(interleaved, f32, T):
    """Bit for bit: an infinity or a NaN of any kind stays in its channel, and a zero keeps its sign.  (300 x 55 heads of 32: two
    pairs a thread in halves of bf16.)"""
    plan = P.rope_plan((16, 16), interleaved=interleaved)
    plan.axis[3], plan.axis[8], plan.axis[9] = 2, -1, 7
    H = 3 if T == 5 else 55
    x, pos = _x(T, H, 32, f32, T), _pos(T, 2)
    bits = torch.int32 if f32 else torch.int16
    odd = [0x7F800000, -0x800000, 0x7FC00001, 0x7F810000, -0x7E0000, -2 ** 31, 0, 1, -0x7FFF0000] if f32 else \
        [0x7F80, -0x80, 0x7FC1, 0x7F81, -0x7E, -2 ** 15, 0, 1, -0x7FFF]
    for i in (3, 8, 9):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 16)
        for n, v in enumerate(odd):
            x.view(bits)[n % T, n % H, (a, b)[n % 2]] = v
            x.view(bits)[(n + 1) % T, n // 2 % H, (b, a)[n % 2]] = v
    for y in (P.rope(x, pos, plan), P.rope(x, pos, plan, inverse=True), P.rope(x.clone(), pos, plan, stream=torch.cuda.current_stream())):
        for i in (3, 8, 9):
            at = slice(2 * i, 2 * i + 2) if interleaved else slice(i, i + 17, 16)
            assert torch.equal(y.view(bits)[..., at], x.view(bits)[..., at])


def test_what_is_not_finite():
    """It stays in its pair; a NaN position, in its token's pairs of that axis."""
    plan = P.rope_plan((16, 16), interleaved=True)
    x, pos = _x(6, 3, 32), _pos(6, 2, True)
    want = P.rope(x, pos, plan)
    bad = x.clone()
    bad[2, 1, 5], bad[4, 0, 30] = NAN, INF
    got = P.rope(bad, pos, plan)
    assert got[2, 1, 4:6].isnan().all() and not torch.isfinite(got[4, 0, 30:]).any()
    got[2, 1, 4:6], got[4, 0, 30:] = want[2, 1, 4:6], want[4, 0, 30:]
    assert torch.equal(got, want)
    for v in (NAN, INF):
        p = pos.clone()
        p[3, 1] = v
        got = P.rope(x, p, plan)
        assert got[3, :, 16:].isnan().all()
        got[3, :, 16:] = want[3, :, 16:]
        assert torch.equal(got, want)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_slices_places_and_streams(f32, interleaved):
    """x as a slice of a wider output, aligned or not, in place, into a given output, on a stream."""
    plan = P.rope_plan((12, 20), interleaved=interleaved)
    pos = _pos(9, 2)
    for start, width in ((0, 400), (32, 416), (1, 403), (4, 404), (2, 402)):
        wide = torch.randn(9, width, generator=torch.Generator().manual_seed(start)).cuda()
        wide = wide if f32 else wide.bfloat16()
        kept, view = wide.clone(), wide[:, start:start + 8 * 40].view(9, 8, 40)
        want = P.rope(view.clone(), pos, plan)
        _check(view, pos, plan, want)
        assert torch.equal(P.rope(view, pos, plan), want)
        assert torch.equal(wide, kept)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        y = P.rope(view, pos, plan, stream=s)
        s.synchronize()
        assert torch.equal(y, want)
        out = torch.full((9, width + 8), 5.0, dtype=view.dtype, device="cuda")
        to = out[:, 8:328].view(9, 8, 40)
        assert P.rope(view, pos, plan, out=to) is to and torch.equal(to, want)
        assert (out[:, :8] == 5).all() and (out[:, 328:] == 5).all()
        assert P.rope(view, pos, plan, out=view) is view and torch.equal(view, want)
        kept[:, start:start + 320] = want.flatten(1)
        assert torch.equal(wide, kept)
    same = _x(1, 8, 40, f32).expand(9, 8, 40)                        # one row for every token
    _check(same, pos, plan, P.rope(same, pos, plan))


def test_turns_undo_each_other():
    for interleaved in (False, True):
        plan = P.rope_plan((44, 42, 42), interleaved=interleaved)
        x, pos = _x(50, 4, 128, True), _pos(50, 3)
        back = P.rope(P.rope(x, pos, plan), pos, plan, inverse=True)
        assert (back - x).abs().max() <= 8 * 2.0 ** -21       # (two turns, each within 2^-22 + 2^-23 + 2^-24 of |x_a| + |x_b| < 8)


def test_many_values():
    """2^32 values in one call, the ends and the middle checked."""
    plan, T, H, D, P_ = P.rope_plan((44, 42, 42), interleaved=True), 2 ** 19, 64, 128, 2 ** 12
    pos = _pos(P_, 3)
    x = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    at = [slice(i, i + 16) for i in (0, T // 2 - 16, T // 2, T - 16)]
    kept = [x[i].clone() for i in at]
    assert P.rope(x, pos, plan, out=x) is x
    for i, w in zip(at, kept):
        _check(w, pos.roll(-i.start, 0)[:16].contiguous(), plan, x[i])
    with pytest.raises(Q.QwamError, match="at most 2\\^32"):
        P.rope(x[:1].expand(T + P_, H, D), pos, plan)
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,dims", [(64, (32,)), (66, (16, 16)), (128, (20, 22, 22)), (67, (32,)), (96, (30, 4))])
def test_large_calls_that_turn_in_part(D, dims, interleaved, f32):
    """2^18 pairs and more, where halves of bf16 take two pairs a thread: the channels behind them stay as they are, into a new
    output, beside other columns and in place."""
    plan = P.rope_plan(dims, interleaved=interleaved)
    T, H = 1100, 17
    assert T * H * sum(dims) // 2 >= 2 ** 18
    x, pos = _x(T, H, D, f32, D), _pos(T // 2, len(dims))
    want = P.rope(x, pos, plan)
    _check(x, pos, plan, want)
    wide = torch.full((T, H * D + 8), 5.0, dtype=x.dtype, device="cuda")
    out = wide[:, 4:4 + H * D].view(T, H, D)
    assert torch.equal(P.rope(x, pos, plan, out=out), want)
    assert (wide[:, :4] == 5).all() and (wide[:, 4 + H * D:] == 5).all()
    assert P.rope(x, pos, plan, out=x) is x and torch.equal(x, want)


# ---- gradients ----

@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_gradient(f32, interleaved, inverse):
    """Against the formula's (the turn back) and against differences: the map is linear, so <g, rope(d)> = <grad, d>."""
    plan = P.rope_plan((20, 22, 22), interleaved=interleaved)
    x, pos, g = _x(30, 3, 80, f32).requires_grad_(), _pos(10, 3), _x(30, 3, 80, f32, 7)
    y = P.rope(x, pos, plan, inverse=inverse)
    assert y.requires_grad
    y.backward(g)
    _check(g, pos, plan, x.grad, not inverse)
    d = _x(30, 3, 80, True, 8)
    moved = _reference(x.detach().double() + d.double(), pos, plan, inverse)[0] - _reference(x.detach(), pos, plan, inverse)[0]
    a, b = float((torch.from_numpy(moved) * g.cpu().double()).sum()), float((x.grad.cpu().double() * d.cpu().double()).sum())
    # 7200 roundings of the gradient, independent, of values and steps of d about 1: 6 deviations of 2^-8 / sqrt 3
    assert abs(a - b) <= 6 * 7200 ** 0.5 * (2.0 ** -8 if not f32 else 2.0 ** -21)


def test_gradient_of_slices_and_shared_rows():
    """Queries and keys beside each other, a gradient that comes transposed, and one row for every token, whose gradients add up."""
    plan, pos = P.rope_plan((32, 32)), _pos(6, 2)
    wide = _x(6, 1, 12 * 64, True)[:, 0].requires_grad_()
    y = P.rope(wide.unflatten(1, (12, 64))[:, :8], pos, plan)
    g = torch.randn(8, 6, 64, generator=torch.Generator().manual_seed(3)).cuda().transpose(0, 1)
    y.backward(g)
    _check(g.contiguous(), pos, plan, wide.grad[:, :512].unflatten(1, (8, 64)).contiguous(), True)
    assert (wide.grad[:, 512:] == 0).all()
    row = _x(1, 8, 64, True).requires_grad_()
    P.rope(row.expand(6, 8, 64), pos, plan).backward(g)
    want = _reference(g.contiguous(), pos, plan, True)[0].sum(0)
    assert np.abs(row.grad[0].cpu().double().numpy() - want).max() <= 6 * 16 * 2.0 ** -21


def test_second_derivative():
    plan, pos = P.rope_plan((16,)), _pos(5, 1)
    x = _x(5, 2, 16, True).requires_grad_()
    y = P.rope(x, pos, plan)
    g, = torch.autograd.grad((y ** 3).sum(), x, create_graph=True)
    h, = torch.autograd.grad((g ** 2).sum() / 2, x)
    r = x.detach().cpu().double().requires_grad_()
    angle = pos.cpu().double() * plan.inv_freq.cpu().double()
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    z = torch.cat((r[..., :8] * c - r[..., 8:] * s, r[..., :8] * s + r[..., 8:] * c), -1)
    rg, = torch.autograd.grad((z ** 3).sum(), r, create_graph=True)
    rh, = torch.autograd.grad((rg ** 2).sum() / 2, r)
    # g = 3 R' y^2 and h = R' 6 y R g in float32: relative errors of a few 2^-21 of sums of magnitudes
    assert float((h.cpu().double() - rh).norm() / rh.norm()) <= 2.0 ** -18


def test_graph_of_a_training_step():
    """Forward and backward in one graph; every replay against eager calls."""
    plan, pos = P.rope_plan((44, 42, 42), interleaved=True), _pos(64, 3)
    x, g = _x(64, 4, 128).requires_grad_(), _x(64, 4, 128, seed=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(P.rope(x, pos, plan), x, g)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = P.rope(x, pos, plan)
        dx, = torch.autograd.grad(y, x, g)
        y = y.detach()
    for i in range(4):
        with torch.no_grad():
            x.copy_(_x(64, 4, 128, seed=20 + i))
        g.copy_(_x(64, 4, 128, seed=40 + i))
        pos.copy_(_pos(64, 3, seed=60 + i))
        y.fill_(NAN)
        dx.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, P.rope(x.detach(), pos, plan)) and torch.equal(dx, P.rope(g, pos, plan, inverse=True)), f"replay {i}"


def test_refusals():
    plan, x, pos = P.rope_plan((16, 16)), _x(6, 3, 32), _pos(6, 2)
    with pytest.raises(Q.QwamError, match="multiple of positions"):
        P.rope(x, pos[:4].contiguous(), plan)
    with pytest.raises(Q.QwamError, match="pairs must be"):
        P.rope(x[..., :30].contiguous(), pos, plan)
    with pytest.raises(Q.QwamError, match="axes must be"):
        P.rope(x, torch.zeros(6, 5, dtype=torch.int32).cuda(), plan)
    with pytest.raises(Q.QwamError, match="heads, dim, positions and tokens must be"):
        P.rope(x[:0], pos, plan)
    with pytest.raises(ValueError, match="positions must be contiguous"):
        P.rope(x, _pos(6, 4)[:, ::2], plan)
    with pytest.raises(ValueError, match="contiguous along its heads"):
        P.rope(_x(6, 6, 32)[:, ::2], pos, plan)
    with pytest.raises(ValueError, match="plan.axis must have shape"):
        P.rope(x, pos, P.RopePlan(plan.inv_freq, plan.axis[:4]))
    with pytest.raises(TypeError, match="plan.inv_freq must be torch.float32"):
        P.rope(x, pos, P.RopePlan(plan.inv_freq.double(), plan.axis))
    with pytest.raises(TypeError, match="out must be torch.bfloat16"):
        P.rope(x, pos, plan, out=x.float())
    with pytest.raises(ValueError, match="out must have shape"):
        P.rope(x, pos, plan, out=x[:3])
    buf = _x(8, 3, 32)
    with pytest.raises(ValueError, match="out overlaps x without being x"):
        P.rope(buf[:6], pos, plan, out=buf[1:7])
    with pytest.raises(Q.QwamError, match="y_stride must be"):
        P.rope(x, pos, plan, out=torch.empty(1, 3, 32, dtype=torch.bfloat16, device="cuda").expand(6, 3, 32))
    leaf = x.clone().requires_grad_()
    for kw in ({"out": torch.empty_like(x)}, {"stream": torch.cuda.current_stream()}):
        with pytest.raises(ValueError, match="takes neither out nor stream"):
            P.rope(leaf, pos, plan, **kw)
    with pytest.raises(ValueError, match="plan.inv_freq requires a gradient, which rope does not have"):
        P.rope(x, pos, P.RopePlan(plan.inv_freq.clone().requires_grad_(), plan.axis))
    with pytest.raises(ValueError, match="positions requires a gradient, which rope does not have"):
        P.rope(x, pos.float().requires_grad_(), plan)
    with pytest.raises(TypeError, match="a bare handle has no pool"):
        P.rope(x, pos, plan, stream=types.SimpleNamespace(cuda_stream=0))
    import torch.autograd.forward_ad as fwd
    with fwd.dual_level(), pytest.raises(ValueError, match="x carries a tangent, which rope does not take on"):
        P.rope(fwd.make_dual(x, torch.ones_like(x)), pos, plan)
    with torch.no_grad():
        assert not P.rope(leaf, pos, plan).requires_grad
