"""The paged key-value cache on the GPU: kv_append against the definition bit for bit, paged_attention against float64.

Bound of an output, derived beforehand: one rounding to bf16 (2^-8 of the value); the weights' two bf16 pieces and the
float32 sums (2^-15 of the weighted magnitudes of V); the scores' float32 error, 2^-20 of the sum of |q k| scale (256
products: a random walk of 16 roundings of 2^-24, and exp's argument), which moves the weights by as much relatively:
    1.01 * 2^-8 |o| + (2^-15 + 2^-19 * max_p scale sum |q k|) * sum_p w |v|.
"""

import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import qwam as Q

pytestmark = pytest.mark.gpu

FP8 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()


def _cache(lengths, H, D, page=16, fp8=False, seed=0, layout="heads", fill=float("nan"), width=None, qscale=1.0):
    """A cache whose sequences hold random keys and values up to `lengths`, `fill` everywhere else."""
    g = torch.Generator().manual_seed(seed)
    used = [-(-max(n, 0) // page) for n in lengths]
    width = max([1] + used) if width is None else width
    total = sum(used) + 2
    order = torch.randperm(total, generator=g)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    kv = torch.full((2, total, H, page, D), fill).bfloat16()
    at = 0
    for b, n in enumerate(lengths):
        table[b, :used[b]] = order[at:at + used[b]].to(torch.int32)
        for i in range(used[b]):
            rows = min(page, n - i * page)
            kv[:, order[at + i], :, :rows] = torch.randn(2, H, rows, D, generator=g).bfloat16()
        at += used[b]
    ks = vs = None
    if fp8:
        kv = (kv.float() * 16).to(FP8)
        ks, vs = (torch.exp(0.3 * torch.randn(H, generator=g)) / 16 for _ in range(2))
    kv = kv.cuda()
    if layout == "rows":                    # pages that hold their rows first
        kv = kv.transpose(2, 3).contiguous().transpose(2, 3)
    k, v = kv[0], kv[1]
    if layout == "both":                    # pages that hold their keys, then their values
        kv = kv.transpose(0, 1).contiguous()
        k, v = kv[:, 0], kv[:, 1]
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    return P.PagedCache(k, v, table.cuda(), dev(ks), dev(vs))


def _q(B, Hq, D, seed=1, scale=1.0):
    return (scale * torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(seed))).bfloat16().cuda()


def _check(cache, q, lengths, out, starts=None, scale=None, max_len=None, least=0.0):
    B, Hq, D = q.shape
    pages, H, page, _ = cache.k.shape
    G = Hq // H
    scale = D ** -0.5 if scale is None else scale
    table = cache.table.cpu()
    reach = table.shape[1] * page
    got = out.cpu().double()
    raw = lambda c: c.float().cpu() if c.dtype == FP8 else c.cpu()  # noqa: E731
    K, V = raw(cache.k).double(), raw(cache.v).double()
    if cache.k_scale is not None:
        K, V = K * cache.k_scale.cpu().double()[:, None, None], V * cache.v_scale.cpu().double()[:, None, None]
    worst = 0.0
    for b in range(B):
        n = max(0, min(int(lengths[b]), reach, reach if max_len is None else max_len))
        lo = 0 if starts is None else max(0, int(starts[b]))
        pos = torch.arange(lo, max(lo, n))
        pg = table[b, pos // page].long() if len(pos) else pos
        ok = (pg >= 0) & (pg < pages)
        pos, pg = pos[ok], pg[ok]
        if not len(pos):
            assert (got[b] == 0).all(), f"sequence {b} sees nothing"
            continue
        k, v = K[pg, :, pos % page], V[pg, :, pos % page]                 # [n][H][D]
        qq = q[b].cpu().double().reshape(H, G, D)
        s = torch.einsum("hgd,nhd->hgn", qq, k) * scale
        sa = torch.einsum("hgd,nhd->hgn", qq.abs(), k.abs()).amax(-1, keepdim=True) * abs(scale)
        w = torch.softmax(s, -1)
        ref = torch.einsum("hgn,nhd->hgd", w, v)
        mag = torch.einsum("hgn,nhd->hgd", w, v.abs())
        e = (got[b].reshape(H, G, D) - ref).abs()
        bound = 1.01 * 2.0 ** -8 * ref.abs() + (2.0 ** -15 + 2.0 ** -19 * sa) * mag + least
        assert torch.isfinite(got[b]).all() and (e <= bound).all(), f"sequence {b} of length {n}: worst {(e / bound).max():.3f} of its bound"
        worst = max(worst, float((e / bound).max()))
    return worst


def _run(lengths, H, G, D, page=16, seed=0, starts=None, **kw):
    cache = _cache(lengths, H, D, page, seed=seed, **kw)
    q = _q(len(lengths), H * G, D, seed + 1)
    L = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    _check(cache, q, lengths, P.paged_attention(cache, q, L, starts=st), starts)


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1023, 1025]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_lengths(D, page, fp8):
    _run(EDGES, 2, 3, D, page, fp8=fp8)


@pytest.mark.parametrize("D", [8, 16, 24, 40, 48, 56, 72, 80, 96, 112, 120, 136, 160, 192, 200, 240, 248, 256])
@pytest.mark.parametrize("fp8", [False, True])
def test_head_widths(D, fp8):
    if fp8 and D % 16:
        pytest.skip("float8 rows come in multiples of 16")
    _run([1, 5, 16, 40, 100, 300, 0, 700], 3, 2, D, 32, fp8=fp8, seed=D)


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 12, 15, 16, 17, 24, 31, 32, 33, 48, 64])
@pytest.mark.parametrize("H", [1, 3])
def test_head_groups(H, G):
    _run([3, 77, 260, 0, 530], H, G, 64, 16, seed=G)
    _run([3, 77, 260, 0, 530], H, G, 128, 16, seed=G, fp8=True)


@pytest.mark.parametrize("layout", ["heads", "rows", "both"])
@pytest.mark.parametrize("fp8", [False, True])
def test_layouts(layout, fp8):
    _run([1, 17, 64, 200, 999], 4, 4, 128, 64, layout=layout, fp8=fp8)
    _run([1, 17, 64, 200, 999], 4, 1, 80, 16, layout=layout, fp8=fp8)


@pytest.mark.parametrize("B,H,L", [(1, 1, 5000), (1, 8, 20000), (2, 1, 70001), (3, 2, 33333), (40, 2, 2000), (1, 16, 77)])
@pytest.mark.parametrize("fp8", [False, True])
def test_long_and_ragged(B, H, L, fp8):
    g = torch.Generator().manual_seed(L)
    lengths = [L] + [int(torch.randint(0, L, (1,), generator=g)) for _ in range(B - 1)]
    _run(lengths, H, 3, 128, 64, fp8=fp8)


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_unwritten_slots(fill):
    for D in (64, 128, 256):
        _run([1, 16, 31, 100, 0, 517], 2, 2, D, 64, fill=fill)


@pytest.mark.parametrize("fp8", [False, True])
def test_starts(fp8):
    lengths = [100, 100, 100, 100, 100, 1000, 1000, 1000, 0, 5]
    starts = [0, 1, 99, 100, 250, 17, 512, 999, 3, -7]
    _run(lengths, 2, 4, 128, 16, starts=starts, fp8=fp8)
    # what lies before a start has no effect, whatever it holds
    cache = _cache(lengths, 2, 128, 16, fp8=fp8)
    q, L, S = _q(len(lengths), 8, 128), torch.tensor(lengths, dtype=torch.int32).cuda(), torch.tensor(starts, dtype=torch.int32).cuda()
    a = P.paged_attention(cache, q, L, starts=S)
    for b, s in enumerate(starts):
        for p in range(0, min(s, lengths[b])):
            page = int(cache.table[b, p // 16])
            for c in (cache.k, cache.v):
                c.view(torch.uint8 if fp8 else torch.int16)[page, :, p % 16] = 0x7F if fp8 else 0x7F80
    assert torch.equal(a, P.paged_attention(cache, q, L, starts=S))


def test_missing_pages_and_limits():
    """Entries outside the pages, lengths past the table and below zero, max_len."""
    lengths = [200, 200, 64, 200, 5000, -3]
    cache = _cache([200, 200, 64, 200, 200, 16], 2, 64, 16, width=13)
    cache.table[0, 3] = -1
    cache.table[1, 0] = cache.k.shape[0]
    cache.table[1, 12] = 2 ** 31 - 1
    cache.table[2, :] = -2 ** 31
    cache.table[3, 4:9] = 10 ** 6
    cache.k.nan_to_num_(0.5)
    cache.v.nan_to_num_(0.5)
    q, L = _q(6, 6, 64), torch.tensor(lengths, dtype=torch.int32).cuda()
    _check(cache, q, lengths, P.paged_attention(cache, q, L))
    for n in (1, 16, 50, 129, 208):
        _check(cache, q, lengths, P.paged_attention(cache, q, L, max_len=n), max_len=n)


@pytest.mark.parametrize("D", [64, 128])
def test_extreme_scores(D):
    """Scores far apart, equal, very negative and with an overflowing neighbour."""
    lengths = [700, 700, 300, 40]
    cache = _cache(lengths, 2, D, 16)
    q = _q(4, 4, D, scale=60.0)
    q[1] = 0
    L = torch.tensor(lengths, dtype=torch.int32).cuda()
    _check(cache, q, lengths, P.paged_attention(cache, q, L))
    _check(cache, q, lengths, P.paged_attention(cache, q, L, scale=-1.0), scale=-1.0)
    _check(cache, q, lengths, P.paged_attention(cache, q, L, scale=0.0), scale=0.0)
    # a constant far below zero on every score: the running maximum starts at nothing, not at a number
    k = torch.where(torch.isnan(cache.k), cache.k, torch.full_like(cache.k, 30.0))
    cache = P.PagedCache(k, cache.v, cache.table)
    _check(cache, -_q(4, 4, D).abs() * 40, lengths, P.paged_attention(cache, -_q(4, 4, D).abs() * 40, L))


def test_query_slices_streams_and_out():
    """q as a slice of a wider layer output; an explicit stream; a given output."""
    lengths = [300, 20, 77]
    cache = _cache(lengths, 2, 64, 32)
    wide = torch.randn(3, 10 * 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    q = wide[:, 64:64 + 8 * 64].view(3, 8, 64)
    L = torch.tensor(lengths, dtype=torch.int32).cuda()
    a = P.paged_attention(cache, q, L)
    _check(cache, q, lengths, a)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = P.paged_attention(cache, q, L, stream=s)
    s.synchronize()
    out = torch.full_like(a, float("nan"))
    assert P.paged_attention(cache, q, L, out=out) is out
    assert torch.equal(a, b) and torch.equal(a, out)


def test_offsets_past_32_bits():
    """Pages more than 2^32 elements apart."""
    H, D, page = 2, 128, 16
    lengths = [40, 100]
    small = _cache(lengths, H, D, page)
    n = small.k.shape[0]
    stride = 2 ** 32 // (n - 1) // 8 * 8 + 8 * H * page * D
    k, v = (torch.empty((n - 1) * stride + H * page * D, dtype=torch.bfloat16, device="cuda")
            .as_strided((n, H, page, D), (stride, page * D, D, 1)) for _ in range(2))
    assert (n - 1) * stride > 2 ** 32
    k.copy_(small.k)
    v.copy_(small.v)
    cache = P.PagedCache(k, v, small.table)
    q, L = _q(2, 6, D), torch.tensor(lengths, dtype=torch.int32).cuda()
    assert torch.equal(P.paged_attention(cache, q, L), P.paged_attention(small, q, L))
    x = torch.randn(2, 2, H, D, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    seq, pos = torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([40, 100], dtype=torch.int32).cuda()
    for c in (cache, small):
        P.kv_append(c, x[0], x[1], seq, pos)
    assert torch.equal(P.paged_attention(cache, q, L + 1), P.paged_attention(small, q, L + 1))
    del k, v, cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fp8", [False, True])
def test_graph(fp8):
    """One graph appends and attends; every replay against eager calls."""
    lengths = [100, 3, 0, 515]
    cache, ref = (_cache([n + 8 for n in lengths], 2, 128, 64, fp8=fp8, width=10) for _ in range(2))
    L = torch.tensor(lengths, dtype=torch.int32).cuda()
    seq = torch.arange(4, dtype=torch.int32).cuda()
    k, v, q = _q(4, 2, 128, 5), _q(4, 2, 128, 6), _q(4, 8, 128, 7)

    def step(c, n):
        P.kv_append(c, k, v, seq, n)
        return P.paged_attention(c, q, n + 1)

    step(ref, L)
    graph = torch.cuda.CUDAGraph()
    n = L.clone()
    with torch.cuda.graph(graph):
        out = step(cache, n)
    for i in range(4):
        n.copy_(L + i)
        for t, s in ((k, 10), (v, 20), (q, 30)):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(s + i)).bfloat16())
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step(ref, L + i)), f"replay {i}"
        _check(cache, q, [m + i + 1 for m in lengths], out)


def test_calls_are_alike():
    lengths = [9000, 100, 4000]
    cache = _cache(lengths, 2, 128, 64)
    q, L = _q(3, 8, 128), torch.tensor(lengths, dtype=torch.int32).cuda()
    a = P.paged_attention(cache, q, L)
    assert all(torch.equal(a, P.paged_attention(cache, q, L)) for _ in range(5))


# ---- append ----

def _bytes(t):
    return t.contiguous().view(torch.uint8) if t.dtype == FP8 else t.contiguous().view(torch.int16)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("layout", ["heads", "rows", "both"])
@pytest.mark.parametrize("H,D,page", [(1, 16, 16), (3, 80, 32), (8, 128, 64), (2, 256, 256)])
def test_append(H, D, page, layout, fp8):
    lengths = [0, 5, 77, 300]
    cache = _cache([n + 40 for n in lengths], H, D, page, fp8=fp8, layout=layout, fill=1.5)
    g = torch.Generator().manual_seed(D)
    seq = torch.tensor([b for b in range(4) for _ in range(37)], dtype=torch.int32)
    pos = torch.tensor([n + i for n in lengths for i in range(37)], dtype=torch.int32)
    perm = torch.randperm(len(seq), generator=g)
    seq, pos = seq[perm], pos[perm]
    seq[3], pos[7], pos[11], seq[13] = -1, -1, 10 ** 6, 4             # tokens without a place
    cache.table[1, (5 + 3) // page] = -1
    wide = (torch.randn(len(seq), 3 * H * D, generator=g) * (8 if fp8 else 1)).bfloat16()
    wide[0, :4] = torch.tensor([448.0, 1e6, -1e6, 0.0])
    wide = wide.cuda()
    k, v = (wide[:, i * H * D:(i + 1) * H * D].view(-1, H, D) for i in (1, 2))
    want = [c.clone() for c in (cache.k, cache.v)]
    table = cache.table.cpu()
    for c, x, s in ((want[0], k, cache.k_scale), (want[1], v, cache.v_scale)):
        y = x if s is None else (x.float() / s[:, None]).clamp(-448, 448).to(FP8)
        y, c = _bytes(y), c.view(torch.uint8 if fp8 else torch.int16)
        for t in range(len(seq)):
            b, p = int(seq[t]), int(pos[t])
            if 0 <= b < 4 and 0 <= p < table.shape[1] * page and 0 <= int(table[b, p // page]) < cache.k.shape[0]:
                c[int(table[b, p // page]), :, p % page] = y[t]
    P.kv_append(cache, k, v, seq.cuda(), pos.cuda())
    for got, ref in zip((cache.k, cache.v), want):
        assert torch.equal(_bytes(got), _bytes(ref))


def test_append_then_attend():
    """Token by token against one call for the whole prompt, and against the definition."""
    H, D, page, n = 2, 64, 16, 50
    x = torch.randn(2, n, H, D, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    a, b = (P.new_cache(6, H, D, 1, 5, page) for _ in range(2))
    for c in (a, b):
        c.table[0, :4] = torch.tensor([5, 0, 2, 3], dtype=torch.int32)
    zero = torch.zeros(n, dtype=torch.int32).cuda()
    pos = torch.arange(n, dtype=torch.int32).cuda()
    P.kv_append(a, x[0], x[1], zero, pos)
    for t in range(n):
        P.kv_append(b, x[0, t:t + 1], x[1, t:t + 1], zero[:1], pos[t:t + 1])
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    q = _q(1, 4, D)
    _check(a, q, [n], P.paged_attention(a, q, torch.tensor([n], dtype=torch.int32).cuda()))


def test_refusals():
    cache = _cache([30, 40], 2, 64, 16)
    q, L = _q(2, 4, 64), torch.tensor([30, 40], dtype=torch.int32).cuda()
    with pytest.raises(Q.QwamError, match="multiple of heads"):
        P.paged_attention(cache, _q(2, 3, 64), L)
    with pytest.raises(Q.QwamError, match="more than 64"):
        P.paged_attention(cache, _q(2, 130, 64), L)
    with pytest.raises(ValueError, match="q must have shape"):
        P.paged_attention(cache, _q(3, 4, 64), L)
    with pytest.raises(TypeError, match="lengths must be torch.int32"):
        P.paged_attention(cache, q, L.long())
    with pytest.raises(ValueError, match="starts must have shape"):
        P.paged_attention(cache, q, L, starts=L[:1])
    with pytest.raises(Q.QwamError, match="max_len must be"):
        P.paged_attention(cache, q, L, max_len=0)
    with pytest.raises(Q.QwamError, match="max_len must be"):
        P.paged_attention(cache, q, L, max_len=49)
    with pytest.raises(Q.QwamError, match="scale must be finite"):
        P.paged_attention(cache, q, L, scale=float("nan"))
    with pytest.raises(ValueError, match="contiguous along its heads"):
        P.paged_attention(cache, _q(2, 8, 64)[:, ::2], L)
    with pytest.raises(TypeError, match="k and v alike"):
        P.paged_attention(P.PagedCache(cache.k, cache.v.half(), cache.table), q, L)
    with pytest.raises(TypeError, match="k_scale must be"):
        P.paged_attention(P.PagedCache(cache.k.to(FP8), cache.v.to(FP8), cache.table), q, L)
    with pytest.raises(Q.QwamError, match="page_size"):
        P.paged_attention(_cache([8], 1, 64, 8), _q(1, 1, 64), L[:1])
    with pytest.raises(Q.QwamError, match="dim must be"):
        P.paged_attention(_cache([8], 1, 60, 16), _q(1, 1, 60), L[:1])
    with pytest.raises(Q.QwamError, match="exceeds 256"):
        P.paged_attention(_cache([8], 1, 264, 16), _q(1, 1, 264), L[:1])
    k = _q(2, 2, 64)
    z = torch.zeros(2, dtype=torch.int32).cuda()
    with pytest.raises(ValueError, match="v must have shape"):
        P.kv_append(cache, k, k[:1], z, z)
    with pytest.raises(TypeError, match="pos must be torch.int32"):
        P.kv_append(cache, k, k, z, z.long())
    with pytest.raises(Q.QwamError, match="tokens must be"):
        P.kv_append(cache, k[:0], k[:0], z[:0], z[:0])
