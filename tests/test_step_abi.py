"""The entry points of a single token's step on the host: bad arguments get their documented status before any HIP call
(the pointers below are fake, never dereferenced)."""

import ctypes
import os

import pytest

from paper_2609_33269_amd import qwam as Q

INVALID, UNSUPPORTED, MISALIGNED = 1, 2, 3
FAKE = 0x10000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(Q.LIB_PATH):
        from paper_2609_33269_amd import build
        build.build()
    return Q.lib()


def _layer(K=256, N=256, r=16, group=64, hadamard=0, **ptrs):
    c = Q.QwamLayerC()
    c.K, c.N, c.r, c.group, c.hadamard = K, N, r, group, hadamard
    for f in ("wq", "ws", "inv_smooth", "L2t", "L1f"):
        setattr(c, f, ptrs.get(f, FAKE))
    c.bias = ptrs.get("bias", None)
    return c


def _matvec(lib, L, M=1, x=FAKE, y=FAKE, ws=FAKE, nbytes=1 << 40):
    return lib.qwam_asp_matvec(ctypes.byref(L), M, x, y, ws, nbytes, None)


def test_matvec_refusals(lib):
    assert lib.qwam_asp_matvec(None, 1, FAKE, FAKE, FAKE, 1 << 40, None) == INVALID
    for kw, st in (({"K": 96}, INVALID), ({"K": 0}, INVALID), ({"N": 24}, INVALID), ({"group": 16}, INVALID),
                   ({"r": 8}, UNSUPPORTED), ({"r": 80}, UNSUPPORTED), ({"r": -16}, UNSUPPORTED),
                   ({"hadamard": 24}, INVALID), ({"K": 131072}, UNSUPPORTED)):
        assert _matvec(lib, _layer(**kw)) == st, kw
        assert lib.qwam_asp_matvec_workspace(ctypes.byref(_layer(**kw)), 1) == -1
    for M, st in ((0, INVALID), (-1, INVALID), (17, UNSUPPORTED)):
        assert _matvec(lib, _layer(), M) == st
        assert lib.qwam_asp_matvec_workspace(ctypes.byref(_layer()), M) == -1
    for f in ("wq", "ws", "L1f", "L2t"):
        assert _matvec(lib, _layer(**{f: None})) == INVALID
        assert _matvec(lib, _layer(**{f: FAKE + 8})) == MISALIGNED
    for f in ("inv_smooth", "bias"):
        assert _matvec(lib, _layer(**{f: FAKE + 2})) == MISALIGNED
    for kw in ("x", "y"):
        assert _matvec(lib, _layer(), **{kw: None}) == INVALID
        assert _matvec(lib, _layer(), **{kw: FAKE + 2}) == MISALIGNED
    need = lib.qwam_asp_matvec_workspace(ctypes.byref(_layer(K=14336, N=256, r=64)), 16)
    if need > 0:
        big = _layer(K=14336, N=256, r=64)
        assert _matvec(lib, big, 16, ws=None) == INVALID
        assert _matvec(lib, big, 16, ws=FAKE + 4) == MISALIGNED
        assert _matvec(lib, big, 16, nbytes=need - 1) == INVALID


def _norm(T=6, D=64, S=2, kind=0, post=0, x_f32=0, eps=1e-6, a=1.0, **ptrs):
    c = Q.QwamNormC()
    c.T, c.D, c.S, c.kind, c.post, c.x_f32, c.eps, c.residual_scale = T, D, S, kind, post, x_f32, eps, a
    for f in ("gate", "scale", "shift", "post_weight", "weight"):
        setattr(c, f, ptrs.get(f, FAKE))
    return c


def _fwd(lib, p, x=FAKE, branch=FAKE, xo=FAKE, h=FAKE):
    return lib.qwam_block_norm(ctypes.byref(p), x, branch, xo, h, None)


def _bwd(lib, p, ws=FAKE, nbytes=1 << 40, **kw):
    names = ("dxo", "dh", "xo", "branch", "dx", "dbranch", "dgate", "dscale", "dshift", "dpost_weight", "dweight")
    return lib.qwam_block_norm_backward(ctypes.byref(p), *(kw.get(n, FAKE) for n in names), ws, nbytes, None)


def test_norm_refusals(lib):
    assert lib.qwam_block_norm(None, FAKE, FAKE, FAKE, FAKE, None) == INVALID
    inf = float("inf")
    for kw, st in (({"T": 0}, INVALID), ({"T": 5}, INVALID), ({"S": 0}, INVALID), ({"D": 0}, INVALID), ({"D": 16385}, UNSUPPORTED),
                   ({"T": 1 << 21, "S": 1}, UNSUPPORTED), ({"kind": 2}, INVALID), ({"eps": -1.0}, INVALID), ({"eps": inf}, INVALID),
                   ({"eps": float("nan")}, INVALID), ({"a": inf}, INVALID), ({"gate": FAKE + 1}, MISALIGNED),
                   ({"weight": FAKE + 1}, MISALIGNED)):
        assert _fwd(lib, _norm(**kw)) == st, kw
        assert _bwd(lib, _norm(**{"post": 1, **kw})) == st, kw
    for kw in ("x", "h", "xo"):
        assert _fwd(lib, _norm(), **{kw: None}) == INVALID
        assert _fwd(lib, _norm(), **{kw: FAKE + 1}) == MISALIGNED
    assert _fwd(lib, _norm(x_f32=1), x=FAKE + 2) == MISALIGNED
    assert _fwd(lib, _norm(), branch=None) == INVALID              # x_out without a branch
    for kw in ("dh", "xo", "dx"):
        assert _bwd(lib, _norm(post=1), **{kw: None}) == INVALID
    for kw in ("dgate", "dscale", "dshift", "dpost_weight", "dweight"):
        assert _bwd(lib, _norm(post=1), **{kw: FAKE + 2}) == MISALIGNED
    assert _bwd(lib, _norm(post=0)) == INVALID                     # dpost_weight without a post-norm
    assert _bwd(lib, _norm(post=1), branch=None) == INVALID
    need = lib.qwam_block_norm_backward_workspace(ctypes.byref(_norm()))
    assert need > 0
    assert _bwd(lib, _norm(post=1), ws=None) == INVALID
    assert _bwd(lib, _norm(post=1), ws=FAKE + 8) == MISALIGNED
    assert _bwd(lib, _norm(post=1), nbytes=need - 1) == INVALID
    assert lib.qwam_block_norm_backward_workspace(ctypes.byref(_norm(T=5))) == -1
    many = _norm(T=1 << 20, S=1 << 20, D=256, post=1)                # 2^22 workgroups for the sums
    assert _bwd(lib, many) == UNSUPPORTED and lib.qwam_block_norm_backward_workspace(ctypes.byref(many)) == -1


def _cache(**kw):
    c = Q.QwamCacheC()
    base = dict(pages=10, page_size=16, heads=2, dim=64, type=0, seqs=3, table_width=4, reserved=0, page_stride=2048,
                head_stride=1024, row_stride=64, k=FAKE, v=FAKE, k_scale=None, v_scale=None, table=FAKE)
    for f, val in {**base, **kw}.items():
        setattr(c, f, val)
    return c


def _append(lib, c, n=3, k=FAKE, ks=128, v=FAKE, vs=128, seq=FAKE, pos=FAKE):
    return lib.qwam_kv_append(ctypes.byref(c), n, k, ks, v, vs, seq, pos, None)


def _attend(lib, c, Hq=4, q=FAKE, qs=256, lengths=FAKE, starts=None, max_len=64, scale=0.1, out=FAKE, ws=FAKE, nbytes=1 << 40):
    return lib.qwam_paged_attention(ctypes.byref(c), Hq, q, qs, lengths, starts, max_len, scale, out, ws, nbytes, None)


def test_cache_refusals(lib):
    assert lib.qwam_kv_append(None, 1, FAKE, 0, FAKE, 0, FAKE, FAKE, None) == INVALID
    for kw, st in (({"type": 2}, INVALID), ({"pages": 0}, INVALID), ({"heads": 0}, INVALID), ({"seqs": 0}, INVALID),
                   ({"table_width": 0}, INVALID), ({"page_size": 8}, INVALID), ({"page_size": 48}, INVALID),
                   ({"page_size": 8192}, INVALID), ({"dim": 60}, INVALID), ({"dim": 264}, UNSUPPORTED), ({"dim": 0}, INVALID),
                   ({"type": 1, "dim": 72}, INVALID), ({"reserved": 1}, INVALID), ({"page_stride": 2044}, MISALIGNED),
                   ({"row_stride": 68}, MISALIGNED), ({"table_width": 1 << 28}, UNSUPPORTED), ({"k": None}, INVALID),
                   ({"v": FAKE + 8}, MISALIGNED), ({"table": None}, INVALID), ({"table": FAKE + 2}, MISALIGNED),
                   ({"type": 1}, INVALID), ({"type": 1, "k_scale": FAKE, "v_scale": FAKE + 1}, MISALIGNED)):
        assert _append(lib, _cache(**kw)) == st, kw
        assert _attend(lib, _cache(**kw)) == st, kw


def test_append_refusals(lib):
    c = _cache()
    assert _append(lib, c, n=0) == INVALID
    assert _append(lib, c, n=1 << 30) == UNSUPPORTED
    for kw in ("k", "v", "seq", "pos"):
        assert _append(lib, c, **{kw: None}) == INVALID
        assert _append(lib, c, **{kw: FAKE + 2}) == MISALIGNED
    assert _append(lib, c, ks=100) == MISALIGNED and _append(lib, c, vs=4) == MISALIGNED


def test_attention_refusals(lib):
    c = _cache()
    for kw, st in (({"Hq": 3}, INVALID), ({"Hq": 0}, INVALID), ({"Hq": 130}, UNSUPPORTED), ({"max_len": 0}, INVALID),
                   ({"max_len": 65}, INVALID)):
        assert _attend(lib, c, **kw) == st, kw
        assert lib.qwam_paged_attention_workspace(ctypes.byref(c), kw.get("Hq", 4), kw.get("max_len", 64)) == -1
    assert _attend(lib, c, scale=float("inf")) == INVALID
    assert _attend(lib, c, qs=60) == MISALIGNED
    for kw in ("q", "lengths", "out"):
        assert _attend(lib, c, **{kw: None}) == INVALID
        assert _attend(lib, c, **{kw: FAKE + 2}) == MISALIGNED
    assert _attend(lib, c, starts=FAKE + 2) == MISALIGNED
    assert lib.qwam_last_error().startswith(b"qwam_paged_attention")
    big = _cache(table_width=65536)
    need = lib.qwam_paged_attention_workspace(ctypes.byref(big), 4, 1 << 20)
    assert need >= 0
    if need > 0:
        assert _attend(lib, big, max_len=1 << 20, ws=None) == INVALID
        assert _attend(lib, big, max_len=1 << 20, ws=FAKE + 4) == MISALIGNED
        assert _attend(lib, big, max_len=1 << 20, nbytes=need - 1) == INVALID
