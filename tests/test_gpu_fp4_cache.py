"""The 4-bit key-value cache on the GPU: kv_append's codes and scales against the definition bit for bit, kv_read's values
exactly, paged_attention against float64 with the bound of the bf16 cache (every stored value is a bf16 value, so a bf16
cache that holds them is the reference's)."""

import ctypes
import types

import numpy as np
import pytest
import torch

import paper_2609_33269_amd as P
from paper_2609_33269_amd import qwam as Q
from test_gpu_paged_attention import EDGES, FP8, _check, _q
from test_gpu_paged_attention import _cache as _wide

pytestmark = pytest.mark.gpu

FP4, E8M0 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.lib()


# ---- the format, from its definition ----

def _quantize(x):
    """float64 [..][dim] -> codes uint8 [..][dim] and exponent bytes uint8 [..][dim / 32]."""
    v = x.numpy().reshape(*x.shape[:-1], -1, 32)
    top = np.abs(v).max(-1)
    e = np.full(top.shape, -123)
    for i in range(-122, 126):
        e = np.where(top > 7 * 2.0 ** (i - 1), i, e)
    with np.errstate(invalid="ignore"):
        a = np.abs(v) * 2.0 ** -e[..., None].astype(np.float64)
        near = np.abs(a[..., None] - GRID)
        near[..., 1::2] += 2.0 ** -40                       # of two as near, the even code
    near = np.where(np.isnan(near), 0.0, near)
    code = near.argmin(-1) + 8 * np.signbit(v)
    byte = np.where(np.isfinite(top), e + 127, 255)
    return torch.from_numpy(code.reshape(x.shape).astype(np.uint8)), torch.from_numpy(byte.astype(np.uint8))


def _pack(code):
    return code[..., ::2] | code[..., 1::2] << 4


def _values(codes, scales):
    """Stored codes [pages][heads][page][dim / 2] and scales [pages][heads][dim / 32][page] -> float64 [pages][heads][page][dim]."""
    c, e = codes.contiguous().view(torch.uint8).cpu().numpy(), scales.view(torch.uint8).cpu().numpy()
    full = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1)
    v = np.where(full & 8, -1.0, 1.0) * GRID[full & 7]
    s = np.where(e == 255, NAN, 2.0 ** (e.astype(np.float64) - 127)).swapaxes(2, 3).repeat(32, -1)
    return torch.from_numpy(v * s)


def _cache(lengths, H, D, page=16, seed=0, layout="heads", width=None, junk=255, device="cuda"):
    """Random codes and scales up to `lengths`; everywhere else any codes and the scale `junk`."""
    g = torch.Generator().manual_seed(seed)
    used = [-(-max(n, 0) // page) for n in lengths]
    width = max([1] + used) if width is None else width
    total = sum(used) + 2
    order = torch.randperm(total, generator=g)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    written = torch.zeros(total, page, dtype=torch.bool)
    at = 0
    for b, n in enumerate(lengths):
        table[b, :used[b]] = order[at:at + used[b]].to(torch.int32)
        for i in range(used[b]):
            written[order[at + i], :min(page, n - i * page)] = True
        at += used[b]
    kv = torch.randint(0, 256, (2, total, H, page, D // 2), generator=g, dtype=torch.uint8).to(device)
    if layout == "rows":                    # pages that hold their rows first
        kv = kv.transpose(2, 3).contiguous().transpose(2, 3)
    k, v = kv[0], kv[1]
    if layout == "both":                    # pages that hold their keys, then their values
        kv = kv.transpose(0, 1).contiguous()
        k, v = kv[:, 0], kv[:, 1]
    s = torch.randint(122, 127, (2, total, H, D // 32, page), generator=g, dtype=torch.uint8)
    s = torch.where(written[None, :, None, None], s, torch.tensor(junk, dtype=torch.uint8)).to(device)
    return P.PagedCache(k.view(FP4), v.view(FP4), table.to(device), s[0].view(E8M0), s[1].view(E8M0))


def _as_bf16(cache):
    """The same keys and values in bf16 pages."""
    def wide(c, s):
        v = _values(c, s)
        b = v.bfloat16()
        assert torch.equal(b.double().nan_to_num(7.0), v.nan_to_num(7.0))
        return b.cuda()
    return P.PagedCache(wide(cache.k, cache.k_scale), wide(cache.v, cache.v_scale), cache.table)


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _run(lengths, H, G, D, page=16, seed=0, starts=None, max_len=None, scale=None, least=0.0, **kw):
    cache = _cache(lengths, H, D, page, seed=seed, **kw)
    q = _q(len(lengths), H * G, D, seed + 1)
    out = P.paged_attention(cache, q, _int(lengths), starts=None if starts is None else _int(starts), max_len=max_len, scale=scale)
    return _check(_as_bf16(cache), q, lengths, out, starts, scale=scale, max_len=max_len, least=least)


# ---- attention ----

@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_lengths(D, page):
    _run(EDGES, 2, 3, D, page)


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
def test_head_widths(D):
    _run([1, 5, 16, 40, 100, 300, 0, 700], 3, 2, D, 32, seed=D)
    _run([3000], 1, 5, D, 16, seed=D)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 8, 15, 16, 17, 31, 32, 33, 64])
@pytest.mark.parametrize("H", [1, 3])
def test_head_groups(H, G):
    _run([3, 77, 260, 0, 530], H, G, 64, 16, seed=G)
    _run([3, 77, 260, 0, 530], H, G, 128, 16, seed=G)


@pytest.mark.parametrize("layout", ["heads", "rows", "both"])
def test_layouts(layout):
    for H, G, D, page in ((4, 4, 128, 64), (4, 1, 96, 16), (2, 2, 256, 32), (3, 1, 32, 16)):
        _run([1, 17, 64, 200, 999], H, G, D, page, layout=layout)


@pytest.mark.parametrize("B,H,L", [(1, 1, 5000), (1, 8, 20000), (2, 1, 70001), (40, 2, 2000), (1, 16, 77), (1, 1, 131072)])
def test_long_and_ragged(B, H, L):
    g = torch.Generator().manual_seed(L)
    _run([L] + [int(torch.randint(0, L, (1,), generator=g)) for _ in range(B - 1)], H, 3, 128, 64)


@pytest.mark.parametrize("junk", [0, 1, 200, 252, 255])
def test_unwritten_slots(junk):
    for D in (64, 128, 256):
        _run([1, 16, 31, 100, 0, 517], 2, 2, D, 64, junk=junk)


def test_starts():
    lengths = [100, 100, 100, 100, 100, 1000, 1000, 1000, 0, 5]
    starts = [0, 1, 99, 100, 250, 17, 512, 999, 3, -7]
    for D in (64, 128, 256):
        _run(lengths, 2, 4, D, 16, starts=starts)
    # what lies before a start has no effect, whatever it holds
    cache = _cache(lengths, 2, 128, 16)
    q, L, S = _q(len(lengths), 8, 128), _int(lengths), _int(starts)
    a = P.paged_attention(cache, q, L, starts=S)
    for b, s in enumerate(starts):
        for p in range(0, min(s, lengths[b])):
            for c in (cache.k_scale, cache.v_scale):
                c.view(torch.uint8)[int(cache.table[b, p // 16]), :, :, p % 16] = 255
    assert torch.equal(a, P.paged_attention(cache, q, L, starts=S))


def test_missing_pages_and_limits():
    lengths = [200, 200, 64, 200, 5000, -3]
    cache = _cache([200, 200, 64, 200, 200, 16], 2, 64, 16, width=13, junk=120)
    cache.table[0, 3] = -1
    cache.table[1, 0] = cache.k.shape[0]
    cache.table[1, 12] = 2 ** 31 - 1
    cache.table[2, :] = -2 ** 31
    cache.table[3, 4:9] = 10 ** 6
    q, L, ref = _q(6, 6, 64), _int(lengths), _as_bf16(cache)
    _check(ref, q, lengths, P.paged_attention(cache, q, L))
    for n in (1, 16, 50, 129, 208):
        _check(ref, q, lengths, P.paged_attention(cache, q, L, max_len=n), max_len=n)


def test_scales_of_every_size():
    """Exponents over a wide range, one large, and the smallest that is written, where a result may fall below the normal
    numbers (2^-126) and is taken as 0 or in their steps."""
    lengths = [600]
    cache = _cache(lengths, 2, 128, 16)
    e = torch.randint(60, 150, cache.k_scale.shape, generator=torch.Generator().manual_seed(1), dtype=torch.uint8).cuda()
    cache.k_scale = torch.full_like(e, 100).view(E8M0)
    cache.v_scale = e.view(E8M0)
    q = _q(1, 4, 128)
    _check(_as_bf16(cache), q, lengths, P.paged_attention(cache, q, _int(lengths)))
    for byte in (4, 240):
        cache.v_scale = torch.full_like(e, byte).view(E8M0)
        _check(_as_bf16(cache), q, lengths, P.paged_attention(cache, q, _int(lengths)), least=2.0 ** -126)


def test_extreme_scores():
    """A value of the leading key may be exactly 0, and what the others add to its channel be of any size: a weight below
    2^-126 of the largest, which is 1 before the sums' division, is below float32's normal numbers and may count as 0.  There
    are at most 700, of values of at most 6 / 2: 700 * 3 * 2^-126 < 2^-114 of a result is not held to the bound."""
    lengths = [700, 700, 300, 40]
    for D in (64, 128, 256):
        _run(lengths, 2, 2, D, 16, scale=4.0, least=2.0 ** -114)
        _run(lengths, 2, 2, D, 16, scale=-4.0, least=2.0 ** -114)
        _run(lengths, 2, 2, D, 16, scale=0.0)


@pytest.mark.parametrize("length", [40, 5000])
def test_nan_groups(length):
    """A group without a value (scale byte 255): in a key it makes its head's results NaN, in a value its channels'."""
    cache = _cache([length] * 2, 2, 128, 64)
    q, L = _q(2, 6, 128), _int([length] * 2)
    want = P.paged_attention(cache, q, L)
    page = int(cache.table[1, 0])
    cache.v_scale.view(torch.uint8)[page, 1, 2, 5] = 255
    got = P.paged_attention(cache, q, L)
    assert got[1, 3:, 64:96].isnan().all()
    got[1, 3:, 64:96] = want[1, 3:, 64:96]
    assert torch.equal(got, want)
    cache.v_scale.view(torch.uint8)[page, 1, 2, 5] = 125
    want = P.paged_attention(cache, q, L)
    cache.k_scale.view(torch.uint8)[page, 0, 3, 5] = 255
    got = P.paged_attention(cache, q, L)
    assert got[1, :3].isnan().all()
    got[1, :3] = want[1, :3]
    assert torch.equal(got, want)


def test_query_slices_streams_and_out():
    lengths = [300, 20, 77]
    cache = _cache(lengths, 2, 64, 32)
    wide = torch.randn(3, 10 * 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    q = wide[:, 64:64 + 8 * 64].view(3, 8, 64)
    a = P.paged_attention(cache, q, _int(lengths))
    _check(_as_bf16(cache), q, lengths, a)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = P.paged_attention(cache, q, _int(lengths), stream=s)
    s.synchronize()
    out = torch.full_like(a, NAN)
    assert P.paged_attention(cache, q, _int(lengths), out=out) is out
    assert torch.equal(a, b) and torch.equal(a, out)
    assert all(torch.equal(a, P.paged_attention(cache, q, _int(lengths))) for _ in range(3))


def test_offsets_past_32_bits():
    """Codes' pages more than 2^32 bytes apart, and scales of pages past 2^32 bytes (their codes share one place)."""
    H, D, page, lengths = 2, 128, 16, [40, 100]
    small = _cache(lengths, H, D, page)
    n = small.k.shape[0]
    stride = 2 ** 32 // (n - 1) // 16 * 16 + 16 * H * page * D
    k, v = (torch.empty((n - 1) * stride + H * page * D // 2, dtype=torch.uint8, device="cuda")
            .as_strided((n, H, page, D // 2), (stride, page * D // 2, D // 2, 1)) for _ in range(2))
    k.copy_(small.k.view(torch.uint8))
    v.copy_(small.v.view(torch.uint8))
    far = P.PagedCache(k.view(FP4), v.view(FP4), small.table, small.k_scale.clone(), small.v_scale.clone())
    q, L = _q(2, 6, D), _int(lengths)
    x = torch.randn(2, 2, H, D, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    for c in (far, small):
        P.kv_append(c, x[0], x[1], _int([0, 1]), _int([39, 99]))
    assert torch.equal(P.paged_attention(far, q, L), P.paged_attention(small, q, L))
    at = _int([0, 0, 1, 1]), _int([39, 3, 99, 50])
    assert all(torch.equal(a, b) for a, b in zip(P.kv_read(far, *at), P.kv_read(small, *at)))
    del k, v, far
    torch.cuda.empty_cache()
    pages, page, D = 2 ** 20 + 3, 4096, 32
    codes = torch.randint(0, 256, (2, page, D // 2), generator=torch.Generator().manual_seed(5), dtype=torch.uint8).cuda()
    k, v = (c.as_strided((pages, 1, page, D // 2), (0, 0, D // 2, 1)) for c in codes)
    scales = torch.zeros(pages, 1, 1, page, dtype=torch.uint8, device="cuda")
    scales[pages - 1] = torch.randint(120, 126, (page,), generator=torch.Generator().manual_seed(6), dtype=torch.uint8).cuda()
    far = P.PagedCache(k.view(FP4), v.view(FP4), _int([[pages - 1]]), scales.view(E8M0), scales.view(E8M0))
    near = P.PagedCache(k[:1].view(FP4), v[:1].view(FP4), _int([[0]]), scales[-1:].clone().view(E8M0), scales[-1:].clone().view(E8M0))
    q, L = _q(1, 2, D), _int([4000])
    assert torch.equal(P.paged_attention(far, q, L), P.paged_attention(near, q, L))
    at = _int([0] * 3), _int([0, 1, 4095])
    assert all(torch.equal(a, b) for a, b in zip(P.kv_read(far, *at), P.kv_read(near, *at)))
    x = torch.randn(1, 1, D, generator=torch.Generator().manual_seed(7)).bfloat16().cuda()
    near.k, near.v = k[:1].clone().contiguous(), v[:1].clone().contiguous()
    near.k, near.v = near.k.view(FP4), near.v.view(FP4)
    near.v_scale = near.k_scale
    for c in (far, near):
        P.kv_append(c, x, x, _int([0]), _int([17]))
    assert all(torch.equal(a, b) for a, b in zip(P.kv_read(far, _int([0]), _int([17])), P.kv_read(near, _int([0]), _int([17]))))
    del far, scales
    torch.cuda.empty_cache()


def _two_positions(q, codes):
    """A cache of two positions a sequence, keys of the given codes [sequences][2][D] and values of 1 and -1 throughout: what
    attention gives is tanh of half the difference of the two scores."""
    B, _, D = codes.shape
    k = torch.zeros(B, 1, 16, D // 2, dtype=torch.uint8)
    v = torch.zeros_like(k)
    k[:, 0, :2], v[:, 0, 0], v[:, 0, 1] = _pack(codes.to(torch.uint8)), 0x22, 0xAA
    e = torch.full((B, 1, D // 32, 16), 127, dtype=torch.uint8).cuda().view(E8M0)
    return P.PagedCache(k.cuda().view(FP4), v.cuda().view(FP4), torch.arange(B, dtype=torch.int32)[:, None].cuda(), e, e)


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 256])
@pytest.mark.parametrize("G", [1, 5])
def test_small_products_beside_a_large_one(D, G):
    """A score keeps what lies 2^-14 below the largest product of its channels' neighbourhood: 256 (1 +- 7 * 2^-14), at every place
    of the large channel."""
    q = torch.zeros(D, G, D)
    codes = torch.full((D, 2, D), 2)
    codes[:, 1] = 10                                        # -1
    for b in range(D):
        q[b, :, b // 8 * 8:b // 8 * 8 + 8] = 2.0 ** -14
        q[b, :, b] = 1
        codes[b, 1, b] = 2
    q = q.bfloat16().cuda()
    cache, L = _two_positions(q, codes), _int([2] * D)
    _check(_as_bf16(cache), q, [2] * D, P.paged_attention(cache, q, L, scale=256.0), scale=256.0)


@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("G", [1, 5])
def test_scores_that_nearly_meet(D, G):
    """Two keys out of 96 random ones whose scores are closest: their difference shows the scores' own error."""
    B, g = 512, torch.Generator().manual_seed(D)
    q = torch.randn(B, 1, D, generator=g).bfloat16()
    codes = torch.randint(0, 16, (B, 96, D), generator=g)
    grid = torch.from_numpy(np.concatenate((GRID, -GRID)))
    order = (grid[codes] * q.double()).sum(-1).sort(1)
    i = order.values.diff(dim=1).argmin(1, keepdim=True)
    at = torch.cat((order.indices.gather(1, i), order.indices.gather(1, i + 1)), 1)
    cache, L = _two_positions(q, codes.gather(1, at[..., None].expand(B, 2, D))), _int([2] * B)
    q = q.expand(B, G, D).contiguous().cuda()
    _check(_as_bf16(cache), q, [2] * B, P.paged_attention(cache, q, L, scale=1.0), scale=1.0)


@pytest.mark.parametrize("D,G", [(32, 1), (64, 6), (128, 2), (128, 16), (256, 3)])
def test_an_infinite_query_before_one_key(D, G):
    """It makes that head's result NaN whatever the key holds at its channel: one sign, the other, or 0."""
    codes = torch.full((3, 2, D), 2)
    codes[1, :, 17], codes[2, :, 17] = 10, 0
    cache, L = _two_positions(torch.zeros(3, G, D), codes), _int([1] * 3)
    for bad in (INF, -INF, NAN):
        for scale in (1.0, -1.0):
            q = _q(3, G, D)
            q[:, G // 2, 17] = bad
            got = P.paged_attention(cache, q, L, scale=scale)
            assert got[:, G // 2].isnan().all()
            got[:, G // 2] = 1
            assert (got == 1).all()


FORMS = [(32, 1), (32, 33), (64, 3), (64, 8), (96, 20), (128, 4), (128, 16), (160, 5), (256, 2), (256, 17)]


@pytest.mark.parametrize("D,G", FORMS)
def test_missing_pages_and_limits_of_every_form(D, G):
    lengths = [200, 200, 64, 200, 5000, -3, 700]
    cache = _cache([200, 200, 64, 200, 200, 16, 700], 2, D, 16, width=44, junk=120)
    cache.table[0, 3] = -1
    cache.table[1, 0] = cache.k.shape[0]
    cache.table[1, 12] = 2 ** 31 - 1
    cache.table[2, :] = -2 ** 31
    cache.table[3, 4:9] = 10 ** 6
    cache.table[6, 1:40:3] = -1
    q, L, ref = _q(7, 2 * G, D), _int(lengths), _as_bf16(cache)
    _check(ref, q, lengths, P.paged_attention(cache, q, L))
    for n in (1, 50, 129, 704):
        _check(ref, q, lengths, P.paged_attention(cache, q, L, max_len=n), max_len=n)
    starts = [0, 199, 3, 70, 190, 0, 333]
    _check(ref, q, lengths, P.paged_attention(cache, q, L, starts=_int(starts)), starts)


@pytest.mark.parametrize("length", [40, 3000])
@pytest.mark.parametrize("D,G", FORMS)
def test_nan_groups_of_every_form(D, G, length):
    cache = _cache([length] * 2, 2, D, 64)
    q, L, last = _q(2, 2 * G, D), _int([length] * 2), D // 32 - 1
    want = P.paged_attention(cache, q, L)
    page = int(cache.table[1, 0])
    for place in (0, 5, 39):
        scale = cache.v_scale.view(torch.uint8)[page, 1, last, place].clone()
        cache.v_scale.view(torch.uint8)[page, 1, last, place] = 255
        got = P.paged_attention(cache, q, L)
        assert got[1, G:, 32 * last:].isnan().all()
        got[1, G:, 32 * last:] = want[1, G:, 32 * last:]
        assert torch.equal(got, want)
        cache.v_scale.view(torch.uint8)[page, 1, last, place] = scale
        scale = cache.k_scale.view(torch.uint8)[page, 0, last, place].clone()
        cache.k_scale.view(torch.uint8)[page, 0, last, place] = 255
        got = P.paged_attention(cache, q, L)
        assert got[1, :G].isnan().all()
        got[1, :G] = want[1, :G]
        assert torch.equal(got, want)
        # a start behind it: it has no effect
        after = _int([0, place + 1])
        seen = P.paged_attention(cache, q, L, starts=after)
        cache.k_scale.view(torch.uint8)[page, 0, last, place] = scale
        assert torch.equal(seen, P.paged_attention(cache, q, L, starts=after))


@pytest.mark.parametrize("D,G", FORMS)
def test_rows_that_run_backwards_in_every_form(D, G):
    lengths, H, page = [100, 3, 70, 1200], 3, 16
    cache = _cache(lengths, H, D, page)
    k, v = (c.view(torch.uint8).flip(0, 1, 2).contiguous() for c in (cache.k, cache.v))
    q, L, Hq, reach = _q(4, G * H, D), _int(lengths), G * H, cache.table.shape[1] * page
    want = P.paged_attention(cache, q, L)
    c, lib = cache.c_struct(), Q.lib()
    last = k.numel() - D // 2
    c.k, c.v = k.data_ptr() + last, v.data_ptr() + last
    c.page_stride, c.head_stride, c.row_stride = -H * page * D // 2, -page * D // 2, -D // 2
    out = torch.full_like(want, NAN)
    need = lib.qwam_paged_attention_workspace(ctypes.byref(c), Hq, reach)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    assert need >= 0 and lib.qwam_paged_attention(ctypes.byref(c), Hq, q.data_ptr(), q.stride(0), L.data_ptr(), None, reach, D ** -0.5,
                                                  out.data_ptr(), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, want)


@pytest.mark.parametrize("D,G,H", [(32, 1, 1), (128, 3, 2), (64, 17, 1)])
def test_more_ranges_than_a_grid_dimension(D, G, H):
    """A table past 2^27 positions, nearly empty: what its few pages hold, the last range's among them, as from a table of them alone.
    Its ranges (4096 positions each) are more than 32768."""
    page, width, B = 4096, 32768 + 5, 2
    near = _cache([5 * page - 100, 3 * page - 1], H, D, page)
    far = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = ([0, 16000, 32767, 32768, width - 1], [1, 32766, 32769])
    for b, places in enumerate(at):
        far[b, places] = near.table[b, :len(places)]
    L = _int([width * page - 100, 32770 * page - 1])
    q = _q(B, G * H, D)
    for seqs in ([0, 1], [0], [1]):
        cache = P.PagedCache(near.k, near.v, far[seqs].contiguous(), near.k_scale, near.v_scale)
        small = P.PagedCache(near.k, near.v, near.table[seqs].contiguous(), near.k_scale, near.v_scale)
        assert Q.lib().qwam_paged_attention_workspace(ctypes.byref(cache.c_struct()), G * H, width * page) >= (width - 1) * len(seqs) * G * H * (D + 2) * 4
        _check(_as_bf16(small), q[seqs], [[5 * page - 100, 3 * page - 1][b] for b in seqs], P.paged_attention(cache, q[seqs], L[seqs].contiguous()))


# ---- append ----

@pytest.mark.parametrize("layout", ["heads", "rows", "both"])
@pytest.mark.parametrize("H,D,page", [(1, 32, 16), (3, 96, 32), (8, 128, 64), (2, 256, 256)])
def test_append(H, D, page, layout):
    lengths = [0, 5, 77, 300]
    cache = _cache([n + 40 for n in lengths], H, D, page, layout=layout)
    g = torch.Generator().manual_seed(D)
    seq = torch.tensor([b for b in range(4) for _ in range(37)], dtype=torch.int32)
    pos = torch.tensor([n + i for n in lengths for i in range(37)], dtype=torch.int32)
    perm = torch.randperm(len(seq), generator=g)
    seq, pos = seq[perm], pos[perm]
    seq[3], pos[7], pos[11], seq[13], pos[17] = -1, -1, 10 ** 6, 4, -2 ** 31             # tokens without a place
    cache.table[1, (5 + 3) // page] = -1
    wide = (torch.randn(len(seq), 3 * H * D, generator=g) * torch.exp(3 * torch.randn(len(seq), 1, generator=g))).bfloat16().cuda()
    k, v = (wide[:, i * H * D:(i + 1) * H * D].view(-1, H, D) for i in (1, 2))
    want = [(c.view(torch.uint8).clone(), s.view(torch.uint8).clone()) for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
    table = cache.table.cpu()
    for (c, s), x in zip(want, (k, v)):
        code, byte = _quantize(x.cpu().double())
        code, byte = _pack(code).cuda(), byte.cuda()
        for t in range(len(seq)):
            b, p = int(seq[t]), int(pos[t])
            if 0 <= b < 4 and 0 <= p < table.shape[1] * page and 0 <= int(table[b, p // page]) < cache.k.shape[0]:
                c[int(table[b, p // page]), :, p % page] = code[t]
                s[int(table[b, p // page]), :, :, p % page] = byte[t]
    P.kv_append(cache, k, v, seq.cuda(), pos.cuda())
    for got, scale, (c, s) in zip((cache.k, cache.v), (cache.k_scale, cache.v_scale), want):
        assert torch.equal(got.view(torch.uint8), c) and torch.equal(scale.view(torch.uint8), s)


def _edge_groups():
    """Groups of 32 where the scale or a code can go wrong, as bf16."""
    rows = []
    for top in (7.0, 7.03125, 6.0, 6.9375, 4.0, 3.5, 3.515625, 1.0, 1.75, 1.7578125):
        for e in (-126, -125, -124, -123, -30, 0, 30, 120, 125):
            r = [top, -top, top * 0.96, top / 2, top / 3, -top / 7, top * 2.0 ** -9, 0.0, -0.0]
            rows.append([v * 2.0 ** e if abs(v) * 2.0 ** (e - 127) < 2 else 0.0 for v in r])
    for s in (1.0, 2.0 ** -20, 2.0 ** 20):                       # every border between two codes, and its neighbours
        for sign in (1, -1):
            ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
            rows.append([6.0 * s] + [sign * s * t * f for t in ties for f in (1.0, 1.0 - 2.0 ** -8, 1.0 + 2.0 ** -7)])
    rows += [[0.0], [-0.0] * 32, [2.0 ** -133], [3e38, 1e38], [-3.3895e38, 1.0], [NAN], [1.0, INF], [-INF, 0.0, 1.0], [INF, NAN], [2.0 ** -127] * 32,
             [2.0 ** -120, 2.0 ** -126, 2.0 ** -127]]
    x = torch.zeros(len(rows), 32, dtype=torch.float64)
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r, dtype=torch.float64)
    return x.bfloat16()


def test_append_edges():
    """Largest values at the borders of a power of two, ties, zeros, the range's ends, infinities and NaN."""
    g = _edge_groups()
    n = len(g)
    x = torch.stack((g, g.flip(0), g.roll(7, 1), g.roll(3, 0)), 1).reshape(n, 2, 64)     # 2 heads of 2 groups
    cache = P.new_cache(-(-n // 16), 2, 64, 1, -(-n // 16), 16, FP4)
    cache.table[0] = torch.arange(cache.k.shape[0])
    seq, pos = torch.zeros(n, dtype=torch.int32).cuda(), torch.arange(n, dtype=torch.int32).cuda()
    P.kv_append(cache, x.cuda(), (-x).cuda(), seq, pos)
    k, v = P.kv_read(cache, seq, pos)
    for stored, scale, back, y in ((cache.k, cache.k_scale, k, x), (cache.v, cache.v_scale, v, -x)):
        code, byte = _quantize(y.double())
        there = lambda t: t.transpose(1, 2).reshape(-1, 2, 32)[:n]  # noqa: E731
        got_e = scale.view(torch.uint8).cpu().permute(0, 3, 1, 2).reshape(-1, 2, 2)[:n]
        assert torch.equal(got_e, byte)
        whole = (byte != 255).repeat_interleave(16, -1)
        assert torch.equal(there(stored.view(torch.uint8).cpu())[whole], _pack(code)[whole])
        want = torch.from_numpy(np.where(code & 8, -1.0, 1.0) * GRID[code.numpy() & 7]).double() * torch.where(
            byte == 255, NAN, 2.0 ** (byte.double() - 127)).repeat_interleave(32, -1)
        assert torch.equal(back.cpu().double().nan_to_num(7.0), want.nan_to_num(7.0))


def test_append_then_attend():
    """Token by token against one call for the whole prompt, and against the definition."""
    H, D, page, n = 2, 64, 16, 50
    x = torch.randn(2, n, H, D, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    a, b = (P.new_cache(6, H, D, 1, 5, page, FP4) for _ in range(2))
    for c in (a, b):
        c.table[0, :4] = torch.tensor([5, 0, 2, 3], dtype=torch.int32)
    zero, pos = torch.zeros(n, dtype=torch.int32).cuda(), torch.arange(n, dtype=torch.int32).cuda()
    P.kv_append(a, x[0], x[1], zero, pos)
    for t in range(n):
        P.kv_append(b, x[0, t:t + 1], x[1, t:t + 1], zero[:1], pos[t:t + 1])
    for f in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(a, f).view(torch.uint8), getattr(b, f).view(torch.uint8))
    q = _q(1, 4, D)
    _check(_as_bf16(a), q, [n], P.paged_attention(a, q, _int([n])))
    # stored values are within half a step of the codes, which is at most a seventh of the group's largest
    k, v = P.kv_read(a, zero, pos)
    for got, want in ((k, x[0]), (v, x[1])):
        top = want.float().unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True)
        assert ((got - want).float().unflatten(-1, (-1, 32)).abs() <= top * (2 / 7)).all()


# ---- read ----

@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("layout", ["heads", "rows", "both"])
@pytest.mark.parametrize("H,D,page", [(1, 32, 16), (3, 96, 32), (8, 128, 64), (2, 256, 256)])
def test_read(H, D, page, layout, kind):
    lengths = [0, 5, 77, 300]
    if kind == "fp4":
        cache = _cache(lengths, H, D, page, layout=layout)
        K, V = _values(cache.k, cache.k_scale), _values(cache.v, cache.v_scale)
    else:
        cache = _wide(lengths, H, D, page, fp8=kind == "fp8", layout=layout)
        K, V = cache.k.float().cpu(), cache.v.float().cpu()
        if kind == "fp8":
            K, V = K * cache.k_scale.cpu()[:, None, None], V * cache.v_scale.cpu()[:, None, None]
    cache.table[2, 1:2] = cache.k.shape[0]
    seq, pos = [3] * 300 + [2] * 77 + [1] * 5, list(range(300)) + list(range(77)) + list(range(5))
    seq += [-1, 4, 3, 3, 0, 3, 2 ** 31 - 1]
    pos += [0, 0, -1, 10 ** 6, 0, 2 ** 31 - 1, 2 ** 31 - 1]
    perm = torch.randperm(len(seq), generator=torch.Generator().manual_seed(1)).tolist()
    seq, pos = [seq[i] for i in perm], [pos[i] for i in perm]
    table = cache.table.cpu()
    want = torch.zeros(2, len(seq), H, D, dtype=torch.float64)
    for t, (b, p) in enumerate(zip(seq, pos)):
        if 0 <= b < 4 and 0 <= p < table.shape[1] * page and 0 <= int(table[b, p // page]) < cache.k.shape[0]:
            want[0, t], want[1, t] = K[int(table[b, p // page]), :, p % page], V[int(table[b, p // page]), :, p % page]
    want = want.bfloat16()                    # (fp8: from the float32 product, one rounding; exact for the others)
    same = lambda a, b: torch.equal(a.nan_to_num(7.0).cpu(), b.nan_to_num(7.0))  # noqa: E731
    k, v = P.kv_read(cache, _int(seq), _int(pos))
    assert k.dtype == torch.bfloat16 and k.is_contiguous() and same(k, want[0]) and same(v, want[1])
    # outputs whose rows are apart, and nothing between them touched
    wide = torch.full((len(seq), 3 * H * D + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    out = tuple(wide[:, i * H * D:(i + 1) * H * D].view(-1, H, D) for i in (0, 2))
    got = P.kv_read(cache, _int(seq), _int(pos), out=out)
    assert got[0] is out[0] and got[1] is out[1] and same(out[0], want[0]) and same(out[1], want[1])
    assert (wide[:, H * D:2 * H * D] == 5).all() and (wide[:, 3 * H * D:] == 5).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a, b = P.kv_read(cache, _int(seq), _int(pos), stream=s)
    s.synchronize()
    assert same(a, want[0]) and same(b, want[1])


@pytest.mark.parametrize("first,second", [((0, 128), (128, 128)), ((0, 256), (128, 256)), ((128, 256), (0, 256)), ((136, 384), (0, 384)),
                                          ((0, 256), (7 * 256, 136)), ((0, 512), (128, 256)), ((128, 384), (0, 1152)), ((7 * 256, -256), (128, 256)),
                                          ((7 * 256, -256), (128 + 7 * 256, -256))])
def test_read_into_one_buffer(first, second):
    """Outputs beside each other in one buffer, (element, stride) of each: columns of one matrix, rows in between, either sign; some
    share a row and are refused, the others hold what separate outputs do and leave the rest as it was."""
    H, D, n = 2, 64, 8
    cache = _cache([20], H, D, 16)
    seq, pos = _int([0] * n), _int(list(range(3, 3 + n)))
    want = P.kv_read(cache, seq, pos)
    elements = [torch.cat([torch.arange(128) + at + i * s for i in range(n)]) for at, s in (first, second)]
    buf = torch.full((16384,), 5.0, dtype=torch.bfloat16, device="cuda")
    c, lib = cache.c_struct(), Q.lib()
    st = lib.qwam_kv_read(ctypes.byref(c), n, seq.data_ptr(), pos.data_ptr(), buf.data_ptr() + 2 * first[0], first[1], buf.data_ptr() + 2 * second[0],
                          second[1], torch.cuda.current_stream().cuda_stream)
    ref = torch.full((16384,), 5.0, dtype=torch.bfloat16, device="cuda")
    if len(torch.cat(elements).unique()) < 2 * 128 * n:
        assert st == 1 and lib.qwam_last_error() == b"qwam_kv_read: k and v overlap"
    else:
        assert st == 0
        for e, w in zip(elements, want):
            ref[e.cuda()] = w.flatten()
    assert torch.equal(buf.nan_to_num(7.0), ref.nan_to_num(7.0))


def test_read_of_every_scale():
    """All sixteen codes at every scale byte, among them those that kv_append does not write: exactly the value down to the
    smallest, an infinity past bf16's largest, NaN for 255."""
    cache = P.new_cache(16, 1, 32, 1, 16, 16, FP4)
    cache.table[0] = torch.arange(16)
    codes = torch.arange(16, dtype=torch.uint8).repeat(2)
    for c in (cache.k, cache.v):
        c.view(torch.uint8)[:] = _pack(codes).cuda()
    e = torch.arange(256, dtype=torch.uint8)
    cache.k_scale.view(torch.uint8)[:, 0, 0] = e.view(16, 16).cuda()
    cache.v_scale.view(torch.uint8)[:, 0, 0] = e.flip(0).view(16, 16).cuda()
    k, v = P.kv_read(cache, _int([0] * 256), torch.arange(256, dtype=torch.int32).cuda())
    grid = torch.from_numpy(np.concatenate((GRID, -GRID))).repeat(2)
    for got, b in ((k, e), (v, e.flip(0))):
        want = grid * torch.where(b == 255, NAN, 2.0 ** (b.double() - 127))[:, None]
        want = torch.where(want.abs() >= 2.0 ** 128, want.sign() * INF, want).bfloat16()
        got = got[:, 0].cpu()
        assert torch.equal(got.nan_to_num(7.0, INF, -INF), want.nan_to_num(7.0, INF, -INF))


def _nearest_bf16(x):
    """float64 -> the nearest bf16, ties to even, rounded once."""
    f = x.float()
    e, bits = x - f.double(), f.view(torch.int32)
    away = torch.where(e != 0, torch.where((e > 0) == (x > 0), 1, -1), 0)      # whether |x| lies above or below |f|
    odd = torch.where((bits & 1 == 0) & torch.isfinite(f), away, 0).int()
    return (bits + odd).view(torch.float32).bfloat16()


def test_read_fp8_is_rounded_once():
    """code * scale has up to 28 bits.  Scales that bring one of a code's four odd mantissas next to the middle of two bf16
    values, where its float32 value is the middle itself; the same among results below float32's normal numbers; and the range's
    ends."""
    H, D, page = 16, 256, 16
    scales = [2.0 ** -120, 2.0 ** 118, 1e-38, 3.0, 0.0, 1.0]
    for m in (9, 11, 13, 15):
        for t in (1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 1 + 201 * 2.0 ** -8):
            near = np.float32(t * 16 / m)
            scales += [float(near), float(np.nextafter(near, np.float32(2))), float(np.nextafter(near, np.float32(0)))]
    scales += torch.tensor([0x00AE8B9C, 0x00E1C71C, 0x02064924, 0x02C80005, 0x00EB13B1, 0x00FBBBB8], dtype=torch.int32).view(torch.float32).tolist()
    twice = 0
    for i in range(0, len(scales), H):
        s = torch.tensor(scales[i:i + H], dtype=torch.float32)
        up, down = (torch.arange(256, dtype=torch.uint8).flip(f).expand(1, H, page, D).contiguous().view(FP8) for f in ((), 0))
        cache = P.PagedCache(up.cuda(), down.cuda(), _int([[0]]), s.cuda(), s.flip(0).cuda())
        k, v = P.kv_read(cache, _int([0]), _int([3]))
        for got, c, sc in ((k, up, s), (v, down, s.flip(0))):
            c = c[0, :, 3]
            want = _nearest_bf16(c.double() * sc.double()[:, None])
            twice += int(((c.float() * sc[:, None]).bfloat16() != want)[~want.isnan()].sum())
            assert torch.equal(got[0].cpu().nan_to_num(7.0), want.nan_to_num(7.0))
    assert len(scales) == 48 and twice > 40                # (so many that rounding twice would have shown)


# ---- together ----

def test_graph():
    """One graph turns, appends, attends and reads; every replay against eager calls."""
    lengths, H, D = [100, 3, 0, 515], 2, 128
    cache, ref = (_cache([n + 8 for n in lengths], H, D, 64, width=10) for _ in range(2))
    L, seq = _int(lengths), torch.arange(4, dtype=torch.int32).cuda()
    plan = P.rope_plan((44, 42, 42), interleaved=True)
    qkv = torch.randn(4, (8 + 2 * H) * D, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()

    def step(c, x, n):
        h = x.unflatten(1, (-1, D))
        qk = P.rope(h[:, :8 + H], n[:, None].expand(4, 3).contiguous(), plan)
        P.kv_append(c, qk[:, 8:], h[:, 8 + H:], seq, n)
        return P.paged_attention(c, qk[:, :8], n + 1), *P.kv_read(c, seq, n)

    step(ref, qkv, L)
    graph, n = torch.cuda.CUDAGraph(), L.clone()
    with torch.cuda.graph(graph):
        outs = step(cache, qkv, n)
    for i in range(4):
        n.copy_(L + i)
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(i)).bfloat16())
        for o in outs:
            o.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, step(ref, qkv, L + i)):
            assert torch.equal(o, w), f"replay {i}"
        # what attention saw is what kv_read gives back
        bf, top = P.new_cache(64, H, D, 4, 10, 64), max(lengths) + i + 1
        bf.table[:] = torch.arange(40, dtype=torch.int32).reshape(4, 10)
        sq, ps = torch.arange(4).repeat_interleave(top).int().cuda(), torch.arange(top).repeat(4).int().cuda()
        ps = torch.where(ps <= (L + i)[sq.long()], ps, -1)
        P.kv_append(bf, *P.kv_read(cache, sq, ps), sq, ps)
        qk = P.rope(qkv.unflatten(1, (-1, D))[:, :8 + H], n[:, None].expand(4, 3).contiguous(), plan)
        _check(bf, qk[:, :8], [m + i + 1 for m in lengths], outs[0])


def test_graph_over_a_wide_table():
    """A program records its step with a table for the longest context it will allow, and replays it from the first token on."""
    H, D, page, width = 2, 128, 64, 1024
    lengths = [0, 1, 100, 700, 9000, 5]
    cache = _cache([n + 1 for n in lengths], H, D, page, width=width)
    q, L, ref = _q(len(lengths), 3 * H, D), torch.zeros(len(lengths), dtype=torch.int32, device="cuda"), _as_bf16(cache)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = P.paged_attention(cache, q, L)
    for now in ([0] * 6, [min(n, 1) for n in lengths], lengths, [n // 2 for n in lengths], [0, 1, 100, 5, 700, 5]):
        L.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.paged_attention(cache, q, L)), f"lengths {now}"
        _check(ref, q, now, out)


@pytest.mark.parametrize("lengths", [[1], [100], [1025], [4096], [9000], [20000], [60, 9000, 500, 3000], [4000] * 9, [16385, 16383, 2049, 2047]])
def test_short_contexts_of_wide_tables(lengths):
    """Ranges go by each context, not by the table's reach: whole contexts, windows of them, and a bound on all."""
    for H, G, D in ((1, 3, 128), (2, 5, 64)):
        _run(lengths, H, G, D, 64, width=2048)
        _run(lengths, H, G, D, 64, width=2048, starts=[max(0, n - 1500) for n in lengths])
        _run(lengths, H, G, D, 64, width=2048, max_len=5000)


def test_short_contexts_of_many_rows():
    """Where the sequences' heads fill the chip, a short context stays in one range."""
    _run([500, 1500, 3000, 0, 1, 1024, 1025] * 10, 4, 3, 64, 64, width=512)


def test_refusals():
    cache = _cache([30, 40], 2, 64, 16)
    q, L, z = _q(2, 4, 64), _int([30, 40]), _int([0, 0])
    k = _q(2, 2, 64)
    with pytest.raises(TypeError, match="k_scale must be torch.float8_e8m0fnu"):
        P.paged_attention(P.PagedCache(cache.k, cache.v, cache.table, torch.ones(2).cuda(), torch.ones(2).cuda()), q, L)
    with pytest.raises(ValueError, match="k_scale must have shape"):
        P.kv_append(P.PagedCache(cache.k, cache.v, cache.table, cache.k_scale[:, :, :1], cache.v_scale), k, k, z, L)
    with pytest.raises(TypeError, match="k_scale must be a torch.Tensor"):
        P.kv_read(P.PagedCache(cache.k, cache.v, cache.table), z, L)
    with pytest.raises(ValueError, match="k_scale must be contiguous"):
        s = cache.k_scale.view(torch.uint8).transpose(2, 3).contiguous().transpose(2, 3).view(E8M0)
        P.kv_read(P.PagedCache(cache.k, cache.v, cache.table, s, cache.v_scale), z, L)
    with pytest.raises(ValueError, match="k and v alike"):
        P.kv_read(P.PagedCache(cache.k, cache.v[:1], cache.table, cache.k_scale, cache.v_scale), z, L)
    with pytest.raises(ValueError, match="seq must have shape"):
        P.kv_read(cache, z[:1], L)
    with pytest.raises(TypeError, match="pos must be torch.int32"):
        P.kv_read(cache, z, L.long())
    with pytest.raises(ValueError, match="pos must be a tensor of one dimension"):
        P.kv_read(cache, z, L[:, None])
    with pytest.raises(ValueError, match=r"out\[1\] must have shape"):
        P.kv_read(cache, z, L, out=(k, k[:1]))
    with pytest.raises(TypeError, match=r"out\[0\] must be torch.bfloat16"):
        P.kv_read(cache, z, L, out=(k.float(), k))
    with pytest.raises(Q.QwamError, match="at least heads"):
        P.kv_read(cache, z, L, out=(k[:1].expand(2, 2, 64), k))
    with pytest.raises(Q.QwamError, match="tokens must be"):
        P.kv_read(cache, z[:0], L[:0])
    with pytest.raises(ValueError, match="requires a gradient, which kv_read does not have"):
        P.kv_read(cache, z, L, out=(k, k.clone().requires_grad_()))
    with pytest.raises(ValueError, match="requires a gradient, which kv_append does not have"):
        P.kv_append(cache, k.clone().requires_grad_(), k, z, L)
    with pytest.raises(TypeError, match="a bare handle has no pool"):
        P.kv_read(cache, z, L, stream=types.SimpleNamespace(cuda_stream=0))
    wide = _wide([30, 40], 2, 64, 16, fp8=True)
    wide.k_scale.requires_grad_()
    with pytest.raises(ValueError, match="requires a gradient, which kv_read does not have"):
        P.kv_read(wide, z, L)
    assert wide.k.dtype == FP8


# ---- beyond the ordinary ----

@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("G", [3, 8])
def test_queries_of_unlike_size(D, G):
    """Channels of q up to 2^24 apart within the 32 that share a scale: what lies 2^14 below the largest is held to 2^-22 of
    it, which adds that times the sum of |k| of the 32 channels to a score's error."""
    lengths = [300, 40, 700]
    cache = _cache(lengths, 2, D, 16)
    g = torch.Generator().manual_seed(D)
    q = (torch.randn(3, 2 * G, D, generator=g) * 2.0 ** -torch.randint(0, 25, (3, 2 * G, D), generator=g)).bfloat16().cuda()
    out = P.paged_attention(cache, q, _int(lengths))
    ref = _as_bf16(cache)
    K, V, table = ref.k.cpu().double(), ref.v.cpu().double(), cache.table.cpu()
    for b, n in enumerate(lengths):
        pos = torch.arange(n)
        pg = table[b, pos // 16].long()
        k, v = K[pg, :, pos % 16], V[pg, :, pos % 16]
        qq = q[b].cpu().double().reshape(2, G, D)
        s = torch.einsum("hgd,nhd->hgn", qq, k) * D ** -0.5
        off = 2.0 ** -19 * torch.einsum("hgd,nhd->hgn", qq.abs(), k.abs()) * D ** -0.5
        top = qq.abs().unflatten(-1, (-1, 32)).amax(-1)
        off = (off + 2.0 ** -22 * torch.einsum("hgc,nhc->hgn", top, k.abs().unflatten(-1, (-1, 32)).sum(-1)) * D ** -0.5).amax(-1, keepdim=True)
        w = torch.softmax(s, -1)
        o, mag = torch.einsum("hgn,nhd->hgd", w, v), torch.einsum("hgn,nhd->hgd", w, v.abs())
        e = (out[b].cpu().double().reshape(2, G, D) - o).abs()
        assert (e <= 1.01 * 2.0 ** -8 * o.abs() + (2.0 ** -15 + 2 * off) * mag).all(), f"sequence {b}"


@pytest.mark.parametrize("D,G", [(64, 2), (64, 6), (128, 3), (128, 16), (256, 2)])
def test_queries_that_are_not_finite(D, G):
    """An infinity or NaN makes that head's result NaN, and no other's."""
    lengths = [300, 40]
    cache = _cache(lengths, 2, D, 16)
    q = _q(2, 2 * G, D)
    want = P.paged_attention(cache, q, _int(lengths))
    for bad in (INF, -INF, NAN):
        p = q.clone()
        p[0, 1, 17] = bad
        got = P.paged_attention(cache, p, _int(lengths))
        assert got[0, 1].isnan().all()
        got[0, 1] = want[0, 1]
        assert torch.equal(got, want)
    zero = torch.zeros_like(q)
    _check(_as_bf16(cache), zero, lengths, P.paged_attention(cache, zero, _int(lengths)))
    tiny = (q.float() * 2.0 ** -120).bfloat16()
    _check(_as_bf16(cache), tiny, lengths, P.paged_attention(cache, tiny, _int(lengths)))


def test_rows_that_run_backwards():
    """The C interface takes strides of either sign: pages, heads and rows in the opposite order in memory."""
    import ctypes
    lengths, H, D, page = [100, 3, 70], 3, 128, 16
    cache = _cache(lengths, H, D, page)
    n = cache.k.shape[0]
    k, v = (c.view(torch.uint8).flip(0, 1, 2).contiguous() for c in (cache.k, cache.v))
    q, L = _q(3, 2 * H, D), _int(lengths)
    want = P.paged_attention(cache, q, L)
    c = cache.c_struct()
    last = k.numel() - D // 2
    c.k, c.v = k.data_ptr() + last, v.data_ptr() + last
    c.page_stride, c.head_stride, c.row_stride = -H * page * D // 2, -page * D // 2, -D // 2
    out = torch.full_like(want, NAN)
    lib = Q.lib()
    s = torch.cuda.current_stream().cuda_stream
    assert n > 3 and lib.qwam_paged_attention_workspace(ctypes.byref(c), 2 * H, 112) == 0
    assert lib.qwam_paged_attention(ctypes.byref(c), 2 * H, q.data_ptr(), q.stride(0), L.data_ptr(), None, 112, D ** -0.5, out.data_ptr(), None, 0, s) == 0
    assert torch.equal(out, want)
    seq, pos = _int([0, 1, 2, 2]), _int([99, 2, 0, 69])
    x = torch.randn(2, 4, H, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    P.kv_append(cache, x[0], x[1], seq, pos)
    ke, ve = (e.view(torch.uint8).clone() for e in (cache.k_scale, cache.v_scale))
    c.k_scale, c.v_scale = ke.data_ptr(), ve.data_ptr()
    assert lib.qwam_kv_append(ctypes.byref(c), 4, x[0].data_ptr(), H * D, x[1].data_ptr(), H * D, seq.data_ptr(), pos.data_ptr(), s) == 0
    assert torch.equal(k.flip(0, 1, 2), cache.k.view(torch.uint8)) and torch.equal(v.flip(0, 1, 2), cache.v.view(torch.uint8))
    got = torch.empty_like(x)
    assert lib.qwam_kv_read(ctypes.byref(c), 4, seq.data_ptr(), pos.data_ptr(), got[0].data_ptr(), H * D, got[1].data_ptr(), H * D, s) == 0
    assert all(torch.equal(a, b) for a, b in zip(got, P.kv_read(cache, seq, pos)))


def test_many_tokens():
    """More than 2^31 keys in a call: appended and read back, the ends checked."""
    H, D, page, n = 32, 128, 4096, 2 ** 19 + 5
    pages = -(-n // page)
    cache = P.new_cache(pages, H, D, 1, pages, page, FP4)
    cache.table[0] = torch.arange(pages - 1, -1, -1)
    x = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    seq, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
    P.kv_append(cache, x, x, seq, pos)
    k, v = P.kv_read(cache, seq, pos)
    small = P.new_cache(2, H, D, 1, 1, 64, FP4)
    small.table[0] = 1
    for at in (slice(0, 40), slice(n // 2, n // 2 + 40), slice(n - 40, n)):
        P.kv_append(small, x[at], x[at], seq[:40], pos[:40])
        want, _ = P.kv_read(small, seq[:40], pos[:40])
        assert torch.equal(k[at], want) and torch.equal(v[at], want)
    del x, k, v, cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4"])
def test_read_past_the_caches(kind):
    """Outputs from 144 (4-bit pages) and 256 MiB (fp8) on are written past the caches; the values are those of short calls, on which the tests
    above look, and a kernel behind the call sees them."""
    H, D, page, n = 8, 128, 64, 65536 + 3
    g = torch.Generator(device="cuda").manual_seed(3)
    pages = -(-n // page)
    scale = torch.full((H,), 0.25, device="cuda") if kind == "fp8" else None
    cache = P.new_cache(pages, H, D, 1, pages, page, {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "fp4": FP4}[kind], scale, scale)
    cache.table[0] = torch.randperm(pages, device="cuda", generator=g)
    x = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    seq, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.randperm(n, device="cuda", generator=g).int()
    P.kv_append(cache, x, -x, seq, pos)
    for _ in range(3):
        k, v = P.kv_read(cache, seq, pos)
        total = k + v
        assert not total.any() and k.any()
        for at in range(0, n, 16384):
            a, b = P.kv_read(cache, seq[at:at + 16384], pos[at:at + 16384])
            assert torch.equal(k[at:at + 16384], a) and torch.equal(v[at:at + 16384], b)
    if kind == "bf16":
        assert torch.equal(k, x)
    del x, k, v, total, cache
    torch.cuda.empty_cache()


def test_two_streams():
    """Calls on two streams at once, each with a workspace of its own, and two graphs replayed at once."""
    lengths = [9000, 100, 4000]
    cache = _cache(lengths, 2, 128, 64)
    qs = [_q(3, 8, 128, s) for s in (1, 2)]
    L = _int(lengths)
    want = [P.paged_attention(cache, q, L) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            got[i].append(P.paged_attention(cache, qs[i], L, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(w, g) for w, gs in zip(want, got) for g in gs)
    graphs, outs = [torch.cuda.CUDAGraph() for _ in qs], []
    for graph, q in zip(graphs, qs):
        with torch.cuda.graph(graph):
            outs.append(P.paged_attention(cache, q, L))
    for _ in range(4):
        for o in outs:
            o.fill_(NAN)
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(w, o) for w, o in zip(want, outs))
