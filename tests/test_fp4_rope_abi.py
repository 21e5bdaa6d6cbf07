"""The entry points of the 4-bit cache and of the rotary positions on the host: bad arguments get their documented status
before any HIP call (the pointers below are fake, never dereferenced), and Python names the argument that is wrong."""

import ctypes

import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import qwam as Q
from test_step_abi import FAKE, INVALID, MISALIGNED, UNSUPPORTED, _append, _attend, _cache, lib  # noqa: F401

FP4 = torch.float4_e2m1fn_x2


def _cache4(**kw):
    return _cache(**{**dict(type=4, page_stride=1024, head_stride=512, row_stride=32, k_scale=FAKE, v_scale=FAKE), **kw})


def _read(lib, c, n=3, seq=FAKE, pos=FAKE, k=FAKE, ks=128, v=FAKE, vs=128):  # noqa: F811
    return lib.qwam_kv_read(ctypes.byref(c), n, seq, pos, k, ks, v, vs, None)


@pytest.mark.parametrize("kw,st", [({"type": 3}, INVALID), ({"dim": 48}, INVALID), ({"dim": 16}, INVALID), ({"dim": 288}, UNSUPPORTED),
                                   ({"k_scale": None}, INVALID), ({"v_scale": None}, INVALID), ({"k_scale": FAKE + 4}, MISALIGNED),
                                   ({"v_scale": FAKE + 8}, MISALIGNED), ({"page_stride": 1032}, MISALIGNED), ({"row_stride": 24}, MISALIGNED),
                                   ({"row_stride": 1 << 26}, UNSUPPORTED), ({"k": FAKE + 8}, MISALIGNED), ({"page_size": 24}, INVALID)])
def test_fp4_cache_refusals(lib, kw, st):  # noqa: F811
    c = _cache4(**kw)
    assert _append(lib, c) == st and _attend(lib, c) == st and _read(lib, c) == st


@pytest.mark.parametrize("type_", [0, 1, 4])
def test_read_refusals(lib, type_):  # noqa: F811
    c = {0: _cache(), 1: _cache(type=1, k_scale=FAKE, v_scale=FAKE), 4: _cache4()}[type_]
    assert lib.qwam_kv_read(None, 1, FAKE, FAKE, FAKE, 0, FAKE, 0, None) == INVALID
    assert _read(lib, c, n=0) == INVALID and _read(lib, c, n=-1) == INVALID
    assert _read(lib, c, n=1 << 30) == UNSUPPORTED
    for kw in ("k", "v", "seq", "pos"):
        assert _read(lib, c, **{kw: None}) == INVALID
        assert _read(lib, c, **{kw: FAKE + 2}) == MISALIGNED
    assert _read(lib, c, ks=132) == MISALIGNED and _read(lib, c, vs=132) == MISALIGNED
    # rows of an output that overlap
    for s in (0, 64, -64, 120):
        assert _read(lib, c, ks=s) == INVALID and _read(lib, c, vs=s) == INVALID
    assert lib.qwam_last_error().startswith(b"qwam_kv_read")


def test_read_wants_two_outputs(lib):  # noqa: F811
    for n in (1, 3):
        assert _read(lib, _cache4(), n=n, k=FAKE, v=FAKE) == INVALID
        assert lib.qwam_last_error() == b"qwam_kv_read: k and v are one output"


@pytest.mark.parametrize("n,k,ks,v,vs", [
    (1, 0, 0, 120, 0), (1, 120, 0, 0, 0), (3, 0, 128, 8, 128), (3, 8, 128, 0, 128), (3, 0, 128, 256, 128), (3, 0, 128, 376, 128),
    (3, 0, 256, 120, 256), (3, 128, 256, 8, 256), (3, 0, -128, -256, 128), (3, 256, -128, 0, 128), (3, 0, 256, 632, -256),
    (5, 0, 256, 136, 384), (5, 0, 384, 264, 256), (4, 0, 1 << 40, 3 << 40, 128), (3, 0, 1 << 62, 8, 1 << 62), (100001, 0, 256, 128 + 256 * 100000, -136)])
def test_read_wants_outputs_apart(lib, n, k, ks, v, vs):  # noqa: F811
    """Rows of heads * dim = 128 elements, from element k and v on, ks and vs apart, that share one."""
    at = 1 << 44
    c = _cache4()
    assert c.heads * c.dim == 128
    assert _read(lib, c, n=n, k=at + 2 * k, ks=ks, v=at + 2 * v, vs=vs) == INVALID
    assert lib.qwam_last_error() == b"qwam_kv_read: k and v overlap"


def _plan(**kw):
    c = Q.QwamRopePlanC()
    base = dict(heads=4, dim=64, pairs=32, interleaved=0, axes=3, positions=6, pos_f32=0, x_f32=0, pos=FAKE, inv_freq=FAKE, axis=FAKE)
    for f, val in {**base, **kw}.items():
        setattr(c, f, val)
    return c


def _rope(lib, c, n=6, inverse=0, x=FAKE, xs=256, y=FAKE + (1 << 20), ys=256):  # noqa: F811
    return lib.qwam_rope(ctypes.byref(c), n, inverse, x, xs, y, ys, None)


def test_rope_refusals(lib):  # noqa: F811
    assert lib.qwam_rope(None, 6, 0, FAKE, 256, FAKE, 256, None) == INVALID
    for kw, st in (({"heads": 0}, INVALID), ({"dim": 0}, INVALID), ({"dim": 4097, "pairs": 8}, UNSUPPORTED), ({"pairs": 0}, INVALID), ({"pairs": 33}, INVALID),
                   ({"axes": 0}, INVALID), ({"axes": 5}, INVALID), ({"positions": 0}, INVALID), ({"positions": 4}, INVALID),
                   ({"positions": 12}, INVALID), ({"pos": None}, INVALID), ({"pos": FAKE + 2}, MISALIGNED), ({"inv_freq": None}, INVALID),
                   ({"inv_freq": FAKE + 1}, MISALIGNED), ({"axis": None}, INVALID), ({"axis": FAKE + 2}, MISALIGNED),
                   ({"heads": 1 << 27}, UNSUPPORTED), ({"heads": 2 ** 31 - 1, "dim": 4096}, UNSUPPORTED)):
        assert _rope(lib, _plan(**kw)) == st, kw
    for n in (0, -6):
        assert _rope(lib, _plan(), n=n) == INVALID
    assert _rope(lib, _plan(positions=1), n=2 ** 31 - 1) == UNSUPPORTED
    for kw in ("x", "y"):
        assert _rope(lib, _plan(), **{kw: None}) == INVALID
        assert _rope(lib, _plan(), **{kw: FAKE + 1}) == MISALIGNED
        assert _rope(lib, _plan(x_f32=1), **{kw: FAKE + 2}) == MISALIGNED
    for s in (0, 255, -255, 1):
        assert _rope(lib, _plan(), ys=s) == INVALID
    assert _rope(lib, _plan(), y=FAKE, xs=512, ys=256) == INVALID          # in place with another stride
    assert lib.qwam_last_error().startswith(b"qwam_rope")


def test_python_names_what_is_wrong(lib):  # noqa: F811
    x, pos, plan = torch.zeros(4, 2, 8, dtype=torch.bfloat16), torch.zeros(4, 1, dtype=torch.int32), P.rope_plan((8,), device="cpu")
    with pytest.raises(ValueError, match="positions must be a GPU tensor"):
        P.rope(x, pos, plan)
    with pytest.raises(ValueError, match="x must be a tensor of three dimensions"):
        P.rope(x[0], pos, plan)
    with pytest.raises(TypeError, match="x must be torch.bfloat16 or torch.float32"):
        P.rope(x.half(), pos, plan)
    with pytest.raises(ValueError, match="positions must be a tensor of two dimensions"):
        P.rope(x, pos[:, 0], plan)
    with pytest.raises(TypeError, match="positions must be torch.int32 or torch.float32"):
        P.rope(x, pos.long(), plan)
    with pytest.raises(TypeError, match="plan must be a RopePlan"):
        P.rope(x, pos, (plan.inv_freq, plan.axis))
    for dims in ((), (8, 3), (0,), (8, -2), (4.0,)):
        with pytest.raises(ValueError, match="dims must be positive even integers"):
            P.rope_plan(dims, device="cpu")
    with pytest.raises(ValueError, match="theta must be positive"):
        P.rope_plan((8,), theta=0.0, device="cpu")
    cache = P.new_cache(3, 2, 64, 1, 2, 16, FP4, device="cpu")
    one = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="k must be a GPU tensor"):
        P.kv_read(cache, one, one)
    with pytest.raises(ValueError, match="dim must be a multiple of 32"):
        P.new_cache(3, 2, 48, 1, 2, 16, FP4, device="cpu")


def test_plans():
    plan = P.rope_plan((4, 6, 2), theta=100.0, interleaved=True, device="cpu")
    assert plan.interleaved is True and plan.axis.tolist() == [0, 0, 1, 1, 1, 2]
    want = [1.0, 100.0 ** -0.5, 1.0, 100.0 ** (-1 / 3), 100.0 ** (-2 / 3), 1.0]
    assert plan.inv_freq.dtype == torch.float32 and torch.equal(plan.inv_freq, torch.tensor(want, dtype=torch.float64).float())


def test_new_fp4_cache():
    c = P.new_cache(3, 2, 64, 5, 7, 16, FP4, device="cpu")
    assert c.k.shape == c.v.shape == (3, 2, 16, 32) and c.k.dtype == FP4
    assert c.k_scale.shape == c.v_scale.shape == (3, 2, 2, 16) and (c.k_scale.float() == 1).all() and (c.table == -1).all()
    assert c.k_scale.data_ptr() != c.v_scale.data_ptr() and not c.k.view(torch.uint8).any()
