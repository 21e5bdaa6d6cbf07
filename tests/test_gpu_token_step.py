"""The operators together: two blocks of examples/token_step.py, token by token, against float64 on the CPU from the
dequantized weights.  Each of the ten roundings to bf16 between a step's input and its output is 2^-9 root mean square
relative at most (2^-8 at most, uniform: 2^-8 / sqrt 3), and they are independent: sqrt(10) * 2^-9 = 0.6%; a norm after
each block keeps them from growing.  Bound 1.5%, of the output's norm."""

import importlib.util
import os
import sys

import numpy as np
import pytest
import torch

from oracle import qwam_oracle as O
from paper_2609_33269_amd import qwam as Q

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "token_step.py")


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()
    spec = importlib.util.spec_from_file_location("token_step", PATH)
    m = importlib.util.module_from_spec(spec)
    sys.modules["token_step"] = m
    spec.loader.exec_module(m)
    return m


def _d(t):
    return t.detach().float().cpu().double()


def _weight(layer):
    """[N][K] that acts on unsmoothed x."""
    codes = O.unpack_codes(layer.wq.cpu().numpy()).astype(np.float64)
    w = torch.from_numpy(codes * np.repeat(_d(layer.ws).numpy().T, layer.group, axis=1))
    return (w + _d(layer.L2t) @ _d(layer.L1t)) * _d(layer.inv_smooth)


def _rms(v, w):
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * _d(w)


def _reference(model, x, memory):
    """One step in float64; memory: per block (keys, values) [positions][sequences][key heads][dim] so far, extended here."""
    B, H, KH, D = x.shape[0], model.heads, model.key_heads, model.dim
    h = _rms(x, model.first_norm)
    for b, mem in zip(model.blocks, memory):
        qkv = (h @ _weight(b.qkv).t()).reshape(B, H + 2 * KH, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:]
        mem[0].append(k)
        mem[1].append(v)
        K, V = torch.stack(mem[0]), torch.stack(mem[1])
        s = torch.einsum("bkgd,nbkd->bkgn", q.reshape(B, KH, H // KH, D), K) * D ** -0.5
        a = torch.einsum("bkgn,nbkd->bkgd", torch.softmax(s, -1), V).reshape(B, H * D)
        x = x + _d(b.gate[0]) * (a @ _weight(b.out).t())
        f = torch.nn.functional.gelu(_rms(x, b.norm[0]) @ _weight(b.up).t()) @ _weight(b.down).t()
        x = x + _d(b.gate[1]) * f
        h = _rms(x, b.norm[1])
    return x, h


@pytest.mark.parametrize("B", [1, 3])
def test_steps_against_float64(ex, B):
    model = ex.random_model(2, width=256, ffn=512, heads=4, key_heads=2, seed=B)
    caches = ex.empty_caches(model, B, 20, page=16)
    seq = torch.arange(B, dtype=torch.int32, device="cuda")
    memory = [([], []) for _ in model.blocks]
    g = torch.Generator().manual_seed(7)
    for t in range(18):                                     # past the end of a page
        x = torch.randn(B, model.width, generator=g)
        got = ex.step(model, caches, x.cuda(), seq, torch.full((B,), t, dtype=torch.int32, device="cuda"))
        for name, u, v in zip(("x", "h"), got, _reference(model, x.double(), memory)):
            err = float((_d(u) - v).norm() / v.norm())
            assert err <= 0.015, f"token {t}: {name} {err:.4f}"


def test_graph_replays_equal_eager_steps(ex):
    B = 2
    model = ex.random_model(2, width=256, ffn=512, heads=4, key_heads=2)
    caches, eager = (ex.empty_caches(model, B, 12, page=16) for _ in range(2))
    seq = torch.arange(B, dtype=torch.int32, device="cuda")
    pos, x = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.randn(B, 256, device="cuda")
    ex.step(model, eager, x, seq, pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, h = ex.step(model, caches, x, seq, pos)
    for t in range(6):
        x.copy_(torch.randn(B, 256, generator=torch.Generator().manual_seed(t)))
        pos.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, ex.step(model, eager, x, seq, pos)[1]), f"step {t}"


def test_float8_cache_stays_close(ex):
    """Keys and values within 2^-4 of theirs: the outputs differ, but by less than that."""
    model = ex.random_model(1, width=256, ffn=512, heads=4, key_heads=2)
    a, b = ex.empty_caches(model, 1, 16, page=16), ex.empty_caches(model, 1, 16, page=16, dtype=torch.float8_e4m3fn)
    seq = torch.zeros(1, dtype=torch.int32, device="cuda")
    for t in range(16):
        x = torch.randn(1, 256, generator=torch.Generator().manual_seed(t)).cuda()
        pos = torch.full((1,), t, dtype=torch.int32, device="cuda")
        u, v = ex.step(model, a, x, seq, pos)[0], ex.step(model, b, x, seq, pos)[0]
        assert float((u - v).norm() / u.norm()) <= 2.0 ** -4
