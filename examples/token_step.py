"""One token's step through a stack of transformer blocks on packed 4-bit ASP layers, for up to 16 sequences at once.

A block is, in the library's operators,

    qkv = asp_matvec(block.qkv, h)                         projections on unquantized tokens
    kv_append(cache, k, v, seq, pos)                       the new keys and values into the pages
    a   = paged_attention(cache, q, pos + 1)               attention over everything stored
    x, h = block_norm(x, asp_matvec(block.out, a), ...)    gate, residual, norm in front of the FFN
    f   = asp_matvec(block.down, gelu(asp_matvec(block.up, h)))
    x, h = block_norm(x, f, ...)                           gate, residual, norm in front of the next block

with a float32 residual stream x and everything else bf16.  Weights are random, packed as make_layer packs the layers
of the action expert (1024 channels, 4096 in the FFN, rank 16).  Run as a program, it fills the caches with a prompt,
records a step in a HIP graph and replays it, and prints the time of a step.

    python examples/token_step.py [--blocks 8] [--sequences 4] [--prompt 200] [--steps 64]
"""

from __future__ import annotations

import argparse
import os
import sys
import time
from dataclasses import dataclass
from typing import List

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_33269_amd as qwam  # noqa: E402


@dataclass
class Block:
    qkv: qwam.PackedLayer
    out: qwam.PackedLayer
    up: qwam.PackedLayer
    down: qwam.PackedLayer
    gate: torch.Tensor        # bf16 [2][width]: of the attention's and of the FFN's output
    norm: torch.Tensor        # bf16 [2][width]: weights of the norms in front of the FFN and of the next block


@dataclass
class Model:
    width: int
    heads: int
    key_heads: int
    dim: int
    first_norm: torch.Tensor  # bf16 [width]: in front of the first block
    blocks: List[Block]


def random_layer(K: int, N: int, rank: int, gen: torch.Generator, group: int = 64) -> qwam.PackedLayer:
    """A packed layer of a random weight, its protected basis orthonormal, its smoothing log-normal."""
    W = torch.randn(N, K, generator=gen) / K ** 0.5
    lam = torch.exp(0.3 * torch.randn(K, generator=gen))
    V, _ = torch.linalg.qr(torch.randn(K, rank, generator=gen))
    L1 = V.bfloat16()
    Wt = W * lam
    L2 = (L1.float().t() @ Wt.t()).bfloat16()
    return qwam.make_layer((Wt - (L1.float() @ L2.float()).t()).contiguous().cuda(), lam.cuda(), L1.cuda(), L2.cuda(), group=group)


def random_model(blocks: int, width: int = 1024, ffn: int = 4096, heads: int = 16, key_heads: int = 4, rank: int = 16,
                 seed: int = 0) -> Model:
    g = torch.Generator().manual_seed(seed)
    dim = width // heads
    near_one = lambda *s: (1 + 0.1 * torch.randn(*s, generator=g)).bfloat16().cuda()  # noqa: E731
    layer = lambda K, N: random_layer(K, N, rank, g)  # noqa: E731
    return Model(width, heads, key_heads, dim, near_one(width),
                 [Block(layer(width, (heads + 2 * key_heads) * dim), layer(width, width), layer(width, ffn), layer(ffn, width),
                        0.5 * near_one(2, width), near_one(2, width)) for _ in range(blocks)])


def empty_caches(model: Model, sequences: int, positions: int, page: int = 64, dtype=torch.bfloat16) -> List[qwam.PagedCache]:
    """A cache per block, its pages dealt out to the sequences in turn; the blocks share one table."""
    per = -(-positions // page)
    scale = torch.full((model.key_heads,), 2.0 ** -5, device="cuda") if dtype == torch.float8_e4m3fn else None
    caches = [qwam.new_cache(sequences * per, model.key_heads, model.dim, sequences, per, page, dtype, scale, scale)
              for _ in model.blocks]
    table = torch.arange(sequences * per, dtype=torch.int32, device="cuda").reshape(per, sequences).t().contiguous()
    for c in caches:
        c.table = table
    return caches


def step(model: Model, caches: List[qwam.PagedCache], x: torch.Tensor, seq: torch.Tensor, pos: torch.Tensor):
    """x float32 [sequences][width], the tokens at positions pos (int32) of sequences seq = 0, 1, ..  Returns the
    residual stream behind the last block and its norm."""
    B, H, KH, D = x.shape[0], model.heads, model.key_heads, model.dim
    lengths = pos + 1
    _, h = qwam.block_norm(x, weight=model.first_norm)
    for b, cache in zip(model.blocks, caches):
        qkv = qwam.asp_matvec(b.qkv, h)
        q, k, v = (qkv[:, i:j].unflatten(1, (-1, D)) for i, j in ((0, H * D), (H * D, (H + KH) * D), ((H + KH) * D, (H + 2 * KH) * D)))
        qwam.kv_append(cache, k, v, seq, pos)
        a = qwam.paged_attention(cache, q, lengths)
        x, h = qwam.block_norm(x, qwam.asp_matvec(b.out, a.view(B, H * D)), gate=b.gate[:1], weight=b.norm[0])
        f = qwam.asp_matvec(b.down, torch.nn.functional.gelu(qwam.asp_matvec(b.up, h)))
        x, h = qwam.block_norm(x, f, gate=b.gate[1:], weight=b.norm[1])
    return x, h


def main() -> None:
    p = argparse.ArgumentParser()
    p.add_argument("--blocks", type=int, default=8)
    p.add_argument("--sequences", type=int, default=4)
    p.add_argument("--prompt", type=int, default=200)
    p.add_argument("--steps", type=int, default=64)
    a = p.parse_args()
    model = random_model(a.blocks)
    caches = empty_caches(model, a.sequences, a.prompt + a.steps + 4)
    g = torch.Generator(device="cuda").manual_seed(1)
    seq = torch.arange(a.sequences, dtype=torch.int32, device="cuda")
    # a prompt's keys and values, as prefill would leave them
    n = a.sequences * a.prompt
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    for c in caches:
        k, v = torch.randn(2, n, model.key_heads, model.dim, generator=g, device="cuda").bfloat16()
        qwam.kv_append(c, k, v, at // a.prompt, at % a.prompt)
    x = torch.randn(a.sequences, model.width, generator=g, device="cuda")
    pos = torch.full((a.sequences,), a.prompt, dtype=torch.int32, device="cuda")
    step(model, caches, x, seq, pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, h = step(model, caches, x, seq, pos)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        graph.replay()
        pos += 1
    torch.cuda.synchronize()
    dt = (time.perf_counter() - t) / a.steps
    assert torch.isfinite(h).all()
    print(f"{a.blocks} blocks, {a.sequences} sequences: {dt * 1e6:.1f} us a step, {a.sequences / dt:.0f} tokens/s")


if __name__ == "__main__":
    main()
