"""block_norm and its gradients on the GPU against float64 on the CPU.

Bounds derived beforehand.  h: one rounding to bf16 (2^-8) plus float32 work on
rows of at most 16384 (statistics within 2^-20, a few roundings of 2^-24 of each
quantity that enters): 1.01 * 2^-8 |h| + 2^-17 A, A the sum of the magnitudes
that are added up to h.  x' likewise with its own terms (float32: 2^-21 of
them).  Gradients of rows: 2^-8 (float32: 0) of the value + 2^-17 of the sum of
the magnitudes; sums over rows: 2^-16 of the summed magnitudes.
"""

import itertools

import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import qwam as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()


def _inputs(T, D, S, f32=False, seed=0, mean=0.3):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    bf = lambda t: t.bfloat16().cuda()  # noqa: E731
    x = 2 * n(T, D) + mean
    return {"x": x.cuda() if f32 else bf(x), "branch": bf(n(T, D) - 0.1), "gate": bf(0.5 * n(S, D)), "post_weight": bf(1 + 0.2 * n(D)),
            "weight": bf(1 + 0.2 * n(D)), "scale": bf(0.3 * n(S, D)), "shift": bf(0.3 * n(S, D))}, bf(n(T, D)), n(T, D)


def _d(t):
    return None if t is None else t.detach().cpu().double()


def _unit(v, norm, eps):
    m = v.mean(1, keepdim=True) if norm == "layer" else torch.zeros(v.shape[0], 1, dtype=v.dtype)
    return (v - m) / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + eps), m


def _ref(p, norm, eps, a, post):
    """x', h in the dtype of the inputs' float64 copies, and what bounds their errors."""
    T = p["x"].shape[0]
    S = next((p[n].shape[0] for n in ("gate", "scale", "shift") if p[n] is not None), 1)
    row = torch.arange(T) // (T // S)
    one = torch.ones((), dtype=torch.float64)
    get = lambda n, o: o if p[n] is None else p[n][row] if p[n].dim() == 2 else p[n]  # noqa: E731
    if p["branch"] is None:
        xo, ax = p["x"], p["x"].abs()
    else:
        u, mb = p["branch"], torch.zeros(T, 1, dtype=torch.float64)
        ub = u.abs()
        if post:
            u, mb = _unit(p["branch"], norm, eps)
            r = 1 / torch.sqrt(((p["branch"] - mb) ** 2).mean(1, keepdim=True) + eps)
            ub = (p["branch"].abs() + mb.abs()) * r * get("post_weight", one).abs()
            u = u * get("post_weight", one)
        xo = a * p["x"] + get("gate", one) * u
        ax = (a * p["x"]).abs() + get("gate", one).abs() * ub
    z, m = _unit(xo, norm, eps)
    r = 1 / torch.sqrt(((xo - m) ** 2).mean(1, keepdim=True) + eps)
    f = get("weight", one) * (1 + get("scale", 0 * one))
    h = z * f + get("shift", 0 * one)
    ah = (ax + m.abs()) * r * f.abs() + get("shift", 0 * one).abs()
    return xo, h, ax, ah


def _keep(p, names):
    return {n: (t if n in names or n in ("x", "branch") else None) for n, t in p.items()}


ALL = ("gate", "post_weight", "weight", "scale", "shift")


def _forward_check(p, norm, post, eps=1e-5, a=0.75):
    kw = {n: p[n] for n in ALL if n != "post_weight" or post}
    xo, h = P.block_norm(p["x"], p["branch"], norm=norm, eps=eps, residual_scale=a, post_norm=post, **kw)
    if not post:
        p = {**p, "post_weight": None}
    rx, rh, ax, ah = _ref({n: _d(t) for n, t in p.items()}, norm, eps, a, post)
    f32 = p["x"].dtype == torch.float32
    if p["branch"] is None:
        assert xo is None
    else:
        assert xo.dtype == p["x"].dtype
        e, b = (_d(xo) - rx).abs(), (0 if f32 else 1.01 * 2.0 ** -8) * rx.abs() + 2.0 ** (-21 if f32 and not post else -19) * ax
        assert (e <= b).all(), f"x': worst {(e / b).max():.3f} of its bound"
    e, b = (_d(h) - rh).abs(), 1.01 * 2.0 ** -8 * rh.abs() + 2.0 ** -17 * ah
    assert h.dtype == torch.bfloat16 and (e <= b).all(), f"h: worst {(e / b).max():.3f} of its bound"


WIDTHS = [1, 2, 7, 8, 33, 64, 96, 250, 256, 520, 1000, 1001, 1024, 2048, 2056, 3072, 4095, 4096, 5120, 8192, 8200, 14336, 16383, 16384]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_widths(D, norm):
    for T, S, f32, post in ((6, 3, False, True), (5, 1, True, False)):
        p, _, _ = _inputs(T, D, S, f32, seed=D)
        _forward_check(p, norm, post)


@pytest.mark.parametrize("T,S", [(1, 1), (2, 2), (3, 1), (64, 4), (333, 3), (1024, 2), (4099, 1)])
@pytest.mark.parametrize("f32", [False, True])
def test_rows(T, S, f32):
    for norm, post in (("rms", True), ("layer", False)):
        p, _, _ = _inputs(T, 384, S, f32, seed=T)
        _forward_check(p, norm, post)


@pytest.mark.parametrize("given", list(itertools.chain.from_iterable(itertools.combinations(ALL, k) for k in (0, 1, 4))))
def test_optional_parameters(given):
    p, _, _ = _inputs(12, 200, 3)
    for norm in ("rms", "layer"):
        _forward_check(_keep(p, given), norm, "post_weight" in given)
        _forward_check({**_keep(p, given), "branch": None}, norm, False)
    _forward_check(_keep(p, given), "rms", True)


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_large_mean_and_equal_rows(norm):
    """A mean far above the deviation (the two passes over the row keep it), rows of one value, zero rows."""
    p, _, _ = _inputs(8, 512, 1, True, mean=300.0)
    p["branch"][3] = 0
    p["x"][4] = 2.5
    p["x"][5] = 0
    p["branch"][5] = 0
    p["gate"][:] = 0.25
    p["branch"][4] = 1.0
    _forward_check(p, norm, False, eps=1e-3)
    _forward_check(p, norm, True, eps=1e-3)


def test_slices_of_a_modulation_and_in_place():
    """gate, scale and shift as slices of one wider output; x' written over x; unaligned slices and rows."""
    for D in (256, 257):
        p, _, _ = _inputs(8, D, 2)
        mod = torch.randn(2, 6 * D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
        p["shift"], p["scale"], p["gate"] = (mod[:, i * D:(i + 1) * D] for i in (0, 1, 5))
        _forward_check(p, "layer", False)
        kw = {n: p[n] for n in ("gate", "weight", "scale", "shift")}
        want = P.block_norm(p["x"], p["branch"], norm="rms", **kw)
        x = p["x"].clone()
        h = torch.empty_like(x)
        got = P.block_norm(x, p["branch"], norm="rms", out=(x, h), **kw)
        assert got[0] is x and got[1] is h and torch.equal(x, want[0]) and torch.equal(h, want[1])


# ---- gradients ----

def _grads(p, dxo, dh, norm, eps, a, post):
    """Float64 gradients at the stored x' by the formulas, and the magnitudes that bound their errors."""
    T, D = p["x"].shape
    S = next((p[n].shape[0] for n in ("gate", "scale", "shift") if p[n] is not None), 1)
    row = torch.arange(T) // (T // S)
    one = torch.ones((), dtype=torch.float64)
    get = lambda n, o: o if p[n] is None else p[n][row] if p[n].dim() == 2 else p[n]  # noqa: E731

    def unit_grad(e, v):
        z, m = _unit(v, norm, eps)
        r = 1 / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + eps)
        c = e.mean(1, keepdim=True) if norm == "layer" else 0 * e[:, :1]
        k = (e * z).mean(1, keepdim=True)
        zb = (v.abs() + m.abs()) * r
        return r * (e - c - z * k), z, r, lambda eb: r * (eb + eb.mean(1, keepdim=True) + zb * (eb * zb).mean(1, keepdim=True)), zb

    f = get("weight", one) * (1 + get("scale", 0 * one))
    g, z, r, mag, zb = unit_grad(dh * f, p["x"])
    d, db = dxo + g, dxo.abs() + mag((dh * f).abs())
    alpha = a if p["branch"] is not None else 1.0
    out = {"dx": (alpha * d, abs(alpha) * db)}
    sums = lambda v: torch.zeros(S, D, dtype=torch.float64).index_add_(0, row, v)  # noqa: E731
    A, B = sums(dh * z), sums(dh)
    Am, Bm = sums(dh.abs() * zb), sums(dh.abs())
    w = get("weight", one)
    sc = 1 + p["scale"] if p["scale"] is not None else torch.ones(S, D, dtype=torch.float64)
    out["dscale"], out["dshift"] = (w * A, w.abs() * Am), (B, Bm)
    out["dweight"] = ((sc * A).sum(0), (sc.abs() * Am).sum(0))
    if p["branch"] is not None:
        e, eb = get("gate", one) * d, get("gate", one).abs() * db
        if post:
            wp = get("post_weight", one)
            gb, u, _, magb, ub = unit_grad(e * wp, p["branch"])
            out["dbranch"] = (gb, magb(eb * wp.abs()))
        else:
            u, ub, wp = p["branch"], p["branch"].abs(), one
            out["dbranch"] = (e, eb)
        C, Cm = sums(d * u), sums(db * ub)
        gt = p["gate"] if p["gate"] is not None else torch.ones(S, D, dtype=torch.float64)
        out["dgate"] = (wp * C, wp.abs() * Cm)
        out["dpost_weight"] = ((gt * C).sum(0), (gt.abs() * Cm).sum(0))
    return out


def _backward_check(p, dh, dxo, norm, post, eps=1e-5, a=0.75):
    f32 = p["x"].dtype == torch.float32
    dxo = None if dxo is None else dxo.cuda() if f32 else dxo.bfloat16().cuda()
    if not post:
        p = {**p, "post_weight": None}
    g = P.block_norm_backward(dxo, dh, p["x"], p["branch"], norm=norm, eps=eps, residual_scale=a, post_norm=post,
                              **{n: p[n] for n in ALL})
    q = {n: _d(t) for n, t in p.items()}
    ref = _grads(q, torch.zeros_like(q["x"]) if dxo is None else _d(dxo), _d(dh), norm, eps, a, post)
    for name, got in g.items():
        if got is None:
            assert name == "dbranch" and p["branch"] is None or p.get(name[1:]) is None or p["branch"] is None
            continue
        want, mag = ref[name]
        half = name in ("dx", "dbranch") and got.dtype == torch.bfloat16
        b = (1.01 * 2.0 ** -8 * want.abs() + 2.0 ** -17 * mag) if half else 2.0 ** (-17 if name == "dx" else -16) * mag
        e = (_d(got) - want).abs()
        assert (e <= b + 1e-30).all(), f"{name}: worst {(e / (b + 1e-30)).max():.3f} of its bound"
    return g


@pytest.mark.parametrize("D", [1, 7, 8, 33, 64, 250, 256, 1000, 1001, 2048, 3072, 4095, 8192, 16383, 16384])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_backward_widths(D, norm):
    for T, S, f32, post in ((6, 3, False, True), (5, 1, True, False)):
        p, dh, dxo = _inputs(T, D, S, f32, seed=D)
        _backward_check(p, dh, dxo, norm, post)


@pytest.mark.parametrize("T,S", [(1, 1), (2, 2), (3, 1), (64, 4), (333, 3), (1026, 2), (4099, 1), (520, 520)])
@pytest.mark.parametrize("f32", [False, True])
def test_backward_rows(T, S, f32):
    for norm, post in (("rms", True), ("layer", False), ("layer", True)):
        p, dh, dxo = _inputs(T, 136, S, f32, seed=T)
        _backward_check(p, dh, dxo, norm, post)


@pytest.mark.parametrize("given", list(itertools.chain.from_iterable(itertools.combinations(ALL, k) for k in (0, 1, 4))))
def test_backward_optional_parameters(given):
    p, dh, dxo = _inputs(12, 200, 3)
    for norm in ("rms", "layer"):
        _backward_check(_keep(p, given), dh, dxo, norm, "post_weight" in given)
        _backward_check(_keep(p, given), dh, None, norm, True)
        _backward_check({**_keep(p, given), "branch": None}, dh, dxo, norm, False)


@pytest.mark.parametrize("T,S", [(17, 17), (34, 17), (70000, 70000), (48, 16)])
def test_backward_many_samples(T, S):
    """A gate, scale and shift per row, more samples than a grid's second dimension holds."""
    p, dh, dxo = _inputs(T, 72, S, seed=S)
    _backward_check(p, dh, dxo, "rms", True)


def test_backward_sums_do_not_change():
    p, dh, dxo = _inputs(2048, 520, 2)
    dxo = dxo.bfloat16().cuda()
    call = lambda: P.block_norm_backward(dxo, dh, p["x"], p["branch"], norm="layer", post_norm=True, **{n: p[n] for n in ALL})  # noqa: E731
    a = call()
    for _ in range(3):
        b = call()
        assert all(torch.equal(a[n], b[n]) for n in a)
    only = P.block_norm_backward(dxo, dh, p["x"], p["branch"], norm="layer", post_norm=True, wanted=("dgate",),
                                 **{n: p[n] for n in ALL})
    assert torch.equal(only["dgate"], a["dgate"]) and torch.equal(only["dx"], a["dx"])
    assert all(only[n] is None for n in only if n not in ("dx", "dgate"))


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("post", [False, True])
def test_gradients_against_differences(norm, post):
    """The directional derivative of the float64 forward by central differences (error of order step^2, 1e-7 here)
    against the gradients' inner product, whose bf16 entries are within 2^-8 of their values
    and whose sum, as the roundings are independent, is within 4 * 2^-8 of the root sum of their squares."""
    p, dh, dxo = _inputs(6, 72, 2, f32=True, seed=3)
    a, eps = 0.75, 1e-5
    use = {n: (None if n == "post_weight" and not post else t) for n, t in p.items()}
    xo, _ = P.block_norm(use["x"], use["branch"], norm=norm, eps=eps, residual_scale=a, post_norm=post, **{n: use[n] for n in ALL})
    g = P.block_norm_backward(dxo.cuda(), dh, xo, use["branch"], norm=norm, eps=eps, residual_scale=a, post_norm=post,
                              **{n: use[n] for n in ALL})
    q = {n: _d(t) for n, t in use.items()}
    loss = lambda v: sum((w * o).sum() for w, o in zip((_d(dxo), _d(dh)), _ref(v, norm, eps, a, post)[:2]))  # noqa: E731
    gen = torch.Generator().manual_seed(5)
    for name in q:
        if q[name] is None:
            continue
        v = torch.randn(q[name].shape, generator=gen, dtype=torch.float64)
        step = 1e-4
        diff = (loss({**q, name: q[name] + step * v}) - loss({**q, name: q[name] - step * v})) / (2 * step)
        got = _d(g["d" + name])
        assert abs((got * v).sum() - diff) <= 4 * 2.0 ** -8 * (got * v).square().sum().sqrt() + 1e-4, name


def test_autograd():
    p, dh, dxo = _inputs(64, 264, 2, seed=7)
    leaf = {n: t.clone().requires_grad_() for n, t in p.items()}
    xo, h = P.block_norm(leaf["x"], leaf["branch"], norm="layer", residual_scale=0.5, post_norm=True, **{n: leaf[n] for n in ALL})
    want = P.block_norm(p["x"], p["branch"], norm="layer", residual_scale=0.5, post_norm=True, **{n: p[n] for n in ALL})
    assert torch.equal(xo, want[0]) and torch.equal(h, want[1])
    d = dxo.bfloat16().cuda()
    torch.autograd.backward([xo, h], [d, dh])
    g = P.block_norm_backward(d, dh, xo.detach(), p["branch"], norm="layer", residual_scale=0.5, post_norm=True,
                              **{n: p[n] for n in ALL})
    for n in leaf:
        assert torch.equal(leaf[n].grad, g["d" + n].to(torch.bfloat16)), n
    # only h used, and without a branch
    x = p["x"].clone().requires_grad_()
    _, h = P.block_norm(x, weight=p["weight"])
    h.backward(dh)
    assert torch.equal(x.grad, P.block_norm_backward(None, dh, p["x"], weight=p["weight"])["dx"])
    with pytest.raises(ValueError, match="neither out nor stream"):
        P.block_norm(x, out=(None, torch.empty_like(p["x"])))


def test_streams_and_graph():
    p, dh, dxo = _inputs(70, 264, 2, seed=7)
    d = dxo.bfloat16().cuda()
    kw = dict(norm="layer", post_norm=True, **{n: p[n] for n in ALL})
    run = lambda **k: (*P.block_norm(p["x"], p["branch"], **kw, **k),  # noqa: E731
                       *(P.block_norm_backward(d, dh, p["x"], p["branch"], **kw, **k).values()))
    a = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = run(stream=s)
    s.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in range(4):
        dh.copy_(torch.randn(dh.shape, generator=torch.Generator().manual_seed(i)).bfloat16())
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(out, run())), f"replay {i}"


def test_refusals():
    p, dh, _ = _inputs(6, 64, 2)
    x, b = p["x"], p["branch"]
    with pytest.raises(ValueError, match="norm must be one of"):
        P.block_norm(x, b, norm="batch")
    with pytest.raises(TypeError, match="x must be torch.bfloat16 or"):
        P.block_norm(x.half(), b)
    with pytest.raises(ValueError, match="branch must have shape"):
        P.block_norm(x, b[:3])
    with pytest.raises(ValueError, match="gate must have shape"):
        P.block_norm(x, b, gate=p["gate"][:, :32])
    with pytest.raises(ValueError, match="scale must have shape"):
        P.block_norm(x, b, gate=p["gate"], scale=p["scale"][:1])
    with pytest.raises(ValueError, match="contiguous along its rows"):
        P.block_norm(x, b, gate=p["gate"].t().contiguous().t())
    with pytest.raises(ValueError, match="post_weight without post_norm"):
        P.block_norm(x, b, post_weight=p["post_weight"])
    with pytest.raises(Q.QwamError, match="multiple of S"):
        P.block_norm(x[:5], b[:5], gate=p["gate"])
    with pytest.raises(Q.QwamError, match="eps must be"):
        P.block_norm(x, b, eps=-1.0)
    with pytest.raises(Q.QwamError, match="residual_scale must be finite"):
        P.block_norm(x, b, residual_scale=float("inf"))
    with pytest.raises(Q.QwamError, match="exceeds 16384"):
        P.block_norm(torch.zeros(1, 16385, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError, match="without a branch"):
        P.block_norm(x, out=(torch.empty_like(x), None))
    with pytest.raises(TypeError, match="dx_out must be"):
        P.block_norm_backward(dh.float(), dh, x, b)
    with pytest.raises(ValueError, match="dh must have shape"):
        P.block_norm_backward(None, dh[:1], x, b)
