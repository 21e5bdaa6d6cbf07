"""The performance cases of the rotary positions over several axes and of the 4-bit key-value cache: keys and values quantized
as they are written into the pages, read back, and attended to.

Kinds of cases (field "kind"):
  rope     rope: pairs of a head's channels turned by the token's position on the pair's axis; with "inverse" the gradient
  append   kv_append of new keys and values into 4-bit pages, and kv_read of what was stored for them
  read     kv_read: stored positions of a padded batch as bf16
  attn     paged_attention: one new token per sequence over its 4-bit pages

A 4-bit cache holds groups of 32 channels of a position's head: codes e2m1 (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a
byte, the lower channel in the lower half, and for each group a byte E that stands for 2^(E - 127), 255 for NaN.  A group is
written with the smallest power of two that leaves its largest value at 7 at most (E kept within 4 to 252), each value
divided by it and rounded to the nearest code, ties to the even one, 6 at most.

Where `own` is false, `run` computes the same in elementary torch operations in 32 bits (angles in 64); where it is true it
calls the package.  Inputs are synthetic: bf16 N(0, 1), keys and values with a gain per channel (log-normal), caches whose
unwritten slots hold any code and a NaN scale, as memory that nobody wrote can.
"""
import math
import random

import torch

DEV = "cuda"
own = False

FP4, E8M0 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
GROUP = 32


def listed():
    return [
        # one token of a few sequences, queries and keys of a block beside each other: the smallest call
        _rope("rope_step", 1, 4, 20, 64, (64,), interleaved=False, far=True),
        # two samples of video tokens on one grid of frames, rows and columns, queries and keys of a block
        _rope("rope_video", 2, 4096, 32, 128, (44, 42, 42), interleaved=True),
        # float32 heads turned in part, at fractional times, odd counts
        _rope("rope_odd_f32", 3, 111, 5, 80, (20, 22, 22), interleaved=False, f32=True, frac=True),
        # the gradient of a video batch's queries, in halves
        _rope("rope_gradient", 1, 4096, 24, 128, (32, 48, 48), interleaved=False, inverse=True),
        # one step's keys and values of a batch
        _append("append_step", 16, 1, 8, 128, 64),
        # ragged prompts into an empty cache
        _append("append_prompt", 3, 1365, 8, 128, 32),
        # a short context back, heads of 64
        _read("read_short", 1, 77, 4, 64, 16),
        # ragged contexts as a padded batch
        _read("read_batch", 8, 2048, 8, 128, 64),
        # the action expert's heads over a short context: latency
        _attn("attn_expert", 1, 16, 1, 64, 77, 16),
        # a batch of ragged contexts, three query heads to a key head, one slot of the batch not in use
        _attn("attn_batch", 16, 8, 3, 128, 4096, 64),
        # few wide key heads with many query heads each, in a sliding window
        _attn("attn_window", 5, 2, 16, 256, 20011, 128, window=6001),
        # two long contexts
        _attn("attn_long", 2, 8, 3, 128, 131072, 256),
    ]


def _rope(name, S, rows, heads, dim, dims, interleaved, f32=False, inverse=False, frac=False, far=False):
    return {"name": name, "kind": "rope", "S": S, "rows": rows, "heads": heads, "dim": dim, "axes": len(dims),
            **{"dim%d" % i: d for i, d in enumerate(dims)}, "interleaved": interleaved, "f32": f32, "inverse": inverse, "frac": frac,
            "far": far}


def _append(name, B, L, H, D, page):
    return {"name": name, "kind": "append", "B": B, "L": L, "H": H, "D": D, "page": page}


def _read(name, B, L, H, D, page):
    return {"name": name, "kind": "read", "B": B, "L": L, "H": H, "D": D, "page": page}


def _attn(name, B, H, G, D, L, page, window=0):
    return {"name": name, "kind": "attn", "B": B, "H": H, "G": G, "D": D, "L": L, "page": page, "window": window}


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case of the ranges above: every option of each operator, no case dearer than the largest listed one."""
    kind = rng.choices(["rope", "append", "read", "attn"], [4, 2, 2, 5])[0]
    if kind == "rope":
        axes, f32 = rng.randint(1, 3), rng.random() < 0.3
        while True:
            S, rows, heads = rng.randint(1, 4), round(_log(rng, 1, 8192)), round(_log(rng, 1, 48))
            dim = rng.choice([64, 72, 80, 96, 128, 128, 192, 256])
            if S * rows * heads * dim * (2 if f32 else 1) <= 8192 * 32 * 128:
                break
        pairs = dim // 2 if rng.random() < 0.7 else rng.randint(axes, dim // 2)
        cut = sorted(rng.sample(range(1, pairs), axes - 1))
        dims = tuple(2 * (b - a) for a, b in zip([0] + cut, cut + [pairs]))
        c = _rope("", S, rows, heads, dim, dims, rng.random() < 0.5, f32=f32, inverse=rng.random() < 0.4, frac=rng.random() < 0.3,
                  far=rng.random() < 0.3)
    elif kind in ("append", "read"):
        while True:
            B, H, D = round(_log(rng, 1, 64)), rng.choice([1, 2, 4, 8, 16]), rng.choice([32, 64, 96, 128, 128, 256])
            L = 1 if kind == "append" and rng.random() < 0.4 else round(_log(rng, 1, 8192))
            if B * L * H * D <= 16384 * 8 * 128:
                break
        c = (_append if kind == "append" else _read)("", B, L, H, D, rng.choice([16, 32, 64, 256]))
    else:
        while True:
            B, H, D, L = round(_log(rng, 1, 64)), rng.choice([1, 2, 4, 8, 16]), rng.choice([32, 64, 96, 128, 128, 160, 256]), round(_log(rng, 1, 131072))
            if B * H * D * L <= 1024 * 131072:
                break
        c = _attn("", B, H, rng.choice([1, 2, 3, 4, 6, 8, 16, 32]), D, L, rng.choice([16, 32, 64, 128, 256]),
                  window=rng.choice([0, 0, 0, max(1, L // 3)]))
    del c["name"]
    return c


# ---- inputs, from the seed alone ----

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 1000003)


def _dims(case):
    return [case["dim%d" % i] for i in range(case["axes"])]


def _rope_inputs(case, seed):
    """x, the positions of one sample's tokens, and each pair's frequency and axis."""
    g, rows, axes = _gen(seed), case["rows"], case["axes"]
    x = torch.randn(case["S"] * rows, case["heads"], case["dim"], generator=g, device=DEV).to(torch.float32 if case["f32"] else torch.bfloat16)
    i = torch.arange(rows, device=DEV)
    if case["far"]:                                # tokens of unrelated sequences, far along
        i = torch.randint(0, 1 << 20, (rows,), generator=g, device=DEV)
    side = max(1, round(rows ** 0.4))              # frames of side x side patches
    pos = torch.stack([i] if axes == 1 else [i // side, i % side] if axes == 2 else [i // (side * side), i // side % side, i % side], dim=1)
    pos = pos.float() * 0.37 if case["frac"] else pos.to(torch.int32)
    f = torch.cat([10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d) for d in _dims(case)]).float().to(DEV)
    axis = torch.cat([torch.full((d // 2,), a, dtype=torch.int32) for a, d in enumerate(_dims(case))]).to(DEV)
    return x, pos.contiguous(), f, axis


def _lengths(case):
    """Ragged context lengths of a batch, the same for every seed: the longest first, the second slot of four or more unused."""
    B, L = case["B"], case["L"]
    r = random.Random(B * 1000003 + L)
    n = [L] + [max(1, round(_log(r, max(1, L / 32), L))) for _ in range(B - 1)]
    if B >= 4:
        n[1] = 0
    return n


def _values(shape, g):
    """bf16 [rows][heads][dim] with a gain per channel."""
    gain = torch.exp(0.5 * torch.randn(shape[1:], generator=g, device=DEV))
    return (torch.randn(shape, generator=g, device=DEV) * gain).bfloat16()


def _quantize(x):
    """bf16 [..][dim] -> codes uint8 [..][dim / 2] and scales uint8 [..][dim / 32]."""
    f = x.float().unflatten(-1, (-1, GROUP))
    mant, ex = torch.frexp(f.abs().amax(-1))
    e = (ex - 3 + (mant > 0.875)).clamp(4 - 127, 252 - 127)
    a = torch.ldexp(f.abs(), -e[..., None])
    c = sum((a > t) if odd else (a >= t) for t, odd in ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)))
    c = (c.to(torch.uint8) + 8 * (f < 0).to(torch.uint8)).flatten(-2)
    return c[..., ::2] + 16 * c[..., 1::2], (e + 127).to(torch.uint8)


def _table(case, lengths, g):
    """Tables over pages in a shuffled order, unused entries -1, and the count of pages."""
    P = case["page"]
    used = [-(-n // P) for n in lengths]
    width, total = max(1, max(used)), sum(used) + 1
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b in range(len(lengths)):
        table[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
    return table, total


def _cache(case, lengths, g, filled):
    """Codes and scales in pages: [pages][heads][page][dim / 2] and [pages][heads][dim / 32][page]."""
    H, D, P = case["H"], case["D"], case["page"]
    table, total = _table(case, lengths, g)
    out = []
    for _ in range(2):
        if filled:
            c, s = _quantize(_values((total * P, H, D), g))
            c = c.reshape(total, P, H, D // 2).transpose(1, 2).contiguous()
            s = s.reshape(total, P, H, D // GROUP).permute(0, 2, 3, 1).contiguous()
            written = torch.zeros(total, P, dtype=torch.bool, device=DEV)
            for b, n in enumerate(lengths):
                p = torch.arange(n, device=DEV)
                written[table[b, p // P].long(), p % P] = True
            s = torch.where(written[:, None, None], s, torch.full((), 255, dtype=torch.uint8, device=DEV))
        else:
            c = torch.randint(0, 256, (total, H, P, D // 2), generator=g, device=DEV, dtype=torch.uint8)
            s = torch.full((total, H, D // GROUP, P), 255, dtype=torch.uint8, device=DEV)
        out.append((c, s))
    return {"k": out[0][0], "v": out[1][0], "table": table, "k_scale": out[0][1], "v_scale": out[1][1]}


def _index(counts, firsts, L=None):
    """seq and pos (int32) of counts[b] tokens from firsts[b] on of every sequence, each padded to L tokens of pos -1."""
    seq = [b for b, n in enumerate(counts) for _ in range(n if L is None else L)]
    pos = [(f + i if i < n else -1) for n, f in zip(counts, firsts) for i in range(n if L is None else L)]
    return (torch.tensor(v, dtype=torch.int32, device=DEV) for v in (seq, pos))


def prepare(case, seed):
    k = case["kind"]
    if k == "rope":
        x, pos, f, axis = _rope_inputs(case, seed)
        return {"kind": k, "x": x, "pos": pos, "inv_freq": f, "axis": axis, "interleaved": case["interleaved"], "inverse": case["inverse"]}
    g = _gen(seed)
    if k == "attn":
        n = _lengths(case)
        cache = _cache(case, n, g, True)
        q = torch.randn(case["B"], case["H"] * case["G"], case["D"], generator=g, device=DEV).bfloat16()
        lengths = torch.tensor(n, dtype=torch.int32, device=DEV)
        starts = torch.clamp(lengths - case["window"], min=0) if case["window"] else None
        return {"kind": k, "q": q, "cache": cache, "lengths": lengths, "starts": starts, "scale": case["D"] ** -0.5}
    if k == "read":
        n = _lengths(case)
        cache = _cache(case, n, g, True)
        seq, pos = _index(n, [0] * len(n), case["L"])
        return {"kind": k, "cache": cache, "seq": seq, "pos": pos}
    # a step appends one token to each ragged context; a prompt fills an empty cache
    new = [1] * case["B"] if case["L"] == 1 else _lengths(case)
    before = [37 * b % 512 for b in range(case["B"])] if case["L"] == 1 else [0] * case["B"]
    cache = _cache(case, [a + n for a, n in zip(before, new)], g, False)
    keys, values = (_values((sum(new), case["H"], case["D"]), g) for _ in range(2))
    seq, pos = _index(new, before)
    return {"kind": k, "k": keys, "v": values, "cache": cache, "seq": seq, "pos": pos}


# ---- one pass ----

def _own_run(s):
    import paper_2609_33269_amd as qwam
    k = s["kind"]
    if k == "rope":
        if "handle" not in s:          # the plan that a program keeps for a model
            s["handle"] = qwam.RopePlan(s["inv_freq"], s["axis"], s["interleaved"])
        return qwam.rope(s["x"], s["pos"], s["handle"], inverse=s["inverse"])
    if "handle" not in s:              # the cache object that a program holds
        c = s["cache"]
        s["handle"] = qwam.PagedCache(c["k"].view(FP4), c["v"].view(FP4), c["table"], c["k_scale"].view(E8M0), c["v_scale"].view(E8M0))
    if k == "attn":
        return qwam.paged_attention(s["handle"], s["q"], s["lengths"], starts=s["starts"], scale=s["scale"])
    if k == "append":
        qwam.kv_append(s["handle"], s["k"], s["v"], s["seq"], s["pos"])
    return qwam.kv_read(s["handle"], s["seq"], s["pos"])


def run(s):
    if own:
        return _own_run(s)
    k = s["kind"]
    if k == "rope":
        return _plain_rope(s)
    if k == "attn":
        return _plain_attn(s)
    if k == "append":
        _plain_append(s)
    return _plain_read(s)


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ----

def _plain_rope(s):
    x, pos, f, axis = s["x"], s["pos"], s["inv_freq"], s["axis"]
    (T, _, dim), R = x.shape, 2 * len(f)
    angle = pos.double()[:, axis.long()] * f.double()
    cos, sin = (t.float().repeat(T // len(pos), 1)[:, None] for t in (torch.cos(angle), torch.sin(angle)))
    if s["inverse"]:
        sin = -sin
    v = x.float()
    a, b = (v[..., :R:2], v[..., 1:R:2]) if s["interleaved"] else (v[..., :R // 2], v[..., R // 2:R])
    y = (a * cos - b * sin, a * sin + b * cos)
    y = torch.stack(y, dim=-1).flatten(-2) if s["interleaved"] else torch.cat(y, dim=-1)
    return torch.cat((y, v[..., R:]), dim=-1).to(x.dtype)


def _dequantize(c, e):
    """Codes uint8 [..][dim / 2] and scales uint8 [..][dim / 32] -> float32 [..][dim]."""
    lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=c.device)
    lut = torch.cat((lut, -lut))
    v = torch.stack((lut[(c & 15).int()], lut[(c >> 4).int()]), dim=-1).flatten(-2)
    scale = torch.where(e == 255, math.nan, torch.exp2(e.float() - 127))
    return (v.unflatten(-1, (-1, GROUP)) * scale[..., None]).flatten(-2)


def _plain_append(s):
    c, seq, pos = s["cache"], s["seq"].long(), s["pos"].long()
    P = c["k"].shape[2]
    page, row = c["table"][seq, pos // P].long(), pos % P
    for n in ("k", "v"):
        codes, scales = _quantize(s[n])
        c[n][page, :, row] = codes
        c[n + "_scale"][page, :, :, row] = scales


def _plain_read(s):
    c, seq, pos = s["cache"], s["seq"].long(), s["pos"].long()
    P = c["k"].shape[2]
    there = pos >= 0
    page, row = c["table"][seq, pos.clamp(min=0) // P].long().clamp(min=0), pos.clamp(min=0) % P
    read = lambda n: torch.where(there[:, None, None], _dequantize(c[n][page, :, row], c[n + "_scale"][page, :, :, row]), 0.0)  # noqa: E731
    return read("k").bfloat16(), read("v").bfloat16()


def _plain_attn(s):
    c, q, n = s["cache"], s["q"].float(), s["lengths"]
    (B, Hq, D), (_, H, P, _) = q.shape, c["k"].shape
    at = torch.arange(c["table"].shape[1] * P, device=q.device)
    seen = at[None] < n[:, None]
    if s["starts"] is not None:
        seen = seen & (at[None] >= s["starts"][:, None])
    idx = c["table"].clamp(min=0).long()

    def view(name):                                 # [B][H][positions][D], 0 where nothing is seen
        v = _dequantize(c[name][idx], c[name + "_scale"][idx].transpose(3, 4)).transpose(1, 2).reshape(B, H, -1, D)
        return torch.where(seen[:, None, :, None], v, 0.0)

    x = (q.reshape(B, H, -1, D) * s["scale"]) @ view("k").transpose(2, 3)
    x = torch.where(seen[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    o = (e @ view("v")) / e.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.reshape(B, Hq, D).bfloat16()


# ---- what one pass cannot do without ----

def work(case):
    k = case["kind"]
    if k == "rope":
        n, pairs = case["S"] * case["rows"] * case["heads"] * case["dim"], sum(_dims(case)) // 2
        return {"bytes": 2 * n * (4 if case["f32"] else 2) + 4 * case["rows"] * case["axes"] + 8 * pairs,
                "flops": 6 * case["S"] * case["rows"] * case["heads"] * pairs + 20 * case["rows"] * pairs}
    H, D, n = case["H"], case["D"], _lengths(case)
    row = 2 * H * (D // 2 + D // GROUP)                      # a position's keys and values, stored
    pages = 4 * sum(-(-m // case["page"]) for m in n)
    if k == "attn":
        seen = sum(min(m, case["window"] or m) for m in n)
        return {"bytes": seen * row + 4 * case["B"] * H * case["G"] * D + pages + 4 * case["B"], "flops": 4 * seen * H * case["G"] * D}
    if k == "read":
        return {"bytes": sum(n) * row + case["B"] * case["L"] * (4 * H * D + 8) + pages, "flops": 2 * sum(n) * H * D}
    T = case["B"] if case["L"] == 1 else sum(n)              # in bf16, stored, read and out in bf16
    return {"bytes": T * (8 * H * D + 2 * row + 16), "flops": 8 * T * H * D}


# ---- the same in 64 bits, from the definitions ----

def _exact_rope(case, seed):
    x, pos, f, axis = _rope_inputs(case, seed)
    R = sum(_dims(case))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), torch.stack([pos[:, a] for a in axis.tolist()], dim=1).double() * f.double())
    if case["inverse"]:
        turn = turn.conj()
    y = x.double()
    first, second = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
    for s in range(case["S"]):
        at = slice(s * case["rows"], (s + 1) * case["rows"])
        z = torch.complex(y[at, :, first], y[at, :, second]) * turn[:, None]
        y[at, :, first], y[at, :, second] = z.real, z.imag
    return y


def _exact_stored(x):
    """What the cache holds for x: the nearest of the sixteen values, at each group's power of two."""
    v = x.double().unflatten(-1, (-1, GROUP))
    top = v.abs().amax(-1, keepdim=True)
    step = torch.full_like(top, 2.0 ** -123)
    for e in range(-122, 126):                                # the first power of two with 7 of it at least `top`
        step = torch.where(step * 7 < top, 2.0 ** e, step)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=v.device)
    far = ((v.abs() / step)[..., None] - grid).abs() + 2.0 ** -30 * (torch.arange(8, device=v.device) % 2)    # of two as near, the even code
    return (torch.sign(v) * grid[far.argmin(-1)] * step).flatten(-2)


def _exact_read(c, seq, pos):
    """Position by position through the table; codes as sign, exponent and one bit of mantissa."""
    P = c["k"].shape[2]
    out = []
    for n in ("k", "v"):
        code = torch.stack((c[n] & 15, c[n] >> 4), dim=-1).flatten(-2).double()
        sign, e, m = 1 - 2 * (code // 8), code % 8 // 2, code % 2
        v = sign * torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e - 1))
        v = v * 2.0 ** (c[n + "_scale"].transpose(2, 3).double() - 127).repeat_interleave(GROUP, dim=-1)
        o = torch.zeros(len(seq), *v.shape[1::2], dtype=torch.float64, device=v.device)
        for i, (b, p) in enumerate(zip(seq.tolist(), pos.tolist())):
            if p >= 0:
                o[i] = v[int(c["table_host"][b][p // P]), :, p % P]
        out.append(o)
    return tuple(out)


def _exact_attn(case, seed):
    s = prepare(case, seed)
    c, H, G, D, P = s["cache"], case["H"], case["G"], case["D"], case["page"]
    grid = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12], dtype=torch.float64, device=DEV) / 2
    out = torch.zeros(case["B"], H * G, D, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(case)):
        first = max(0, n - case["window"]) if case["window"] else 0
        pages = c["table"][b, :-(-n // P)].long()
        for h in range(H if first < n else 0):
            kv = []
            for name in ("k", "v"):
                code = c[name][pages, h].reshape(-1, D // 2)[first:n].long()
                value = torch.empty(n - first, D, dtype=torch.float64, device=DEV)
                value[:, 0::2], value[:, 1::2] = grid[code % 16], grid[code // 16]
                e = c[name + "_scale"][pages, h].transpose(1, 2).reshape(-1, D // GROUP)[first:n]
                kv.append(value * (2.0 ** (e.double() - 127)).repeat_interleave(GROUP, dim=1))
            w = torch.softmax(s["q"][b, h * G:(h + 1) * G].double() @ kv[0].t().contiguous() * D ** -0.5, dim=-1)
            out[b, h * G:(h + 1) * G] = w @ kv[1]
    return out


def exact(case, seed):
    k = case["kind"]
    if k == "rope":
        return _exact_rope(case, seed)
    if k == "attn":
        return _exact_attn(case, seed) if case["B"] * case["H"] <= 2048 else None
    s = prepare(case, seed)
    if k == "append":
        return _exact_stored(s["k"]), _exact_stored(s["v"])
    if len(s["seq"]) > 100000:
        return None
    s["cache"]["table_host"] = s["cache"]["table"].tolist()
    return _exact_read(s["cache"], s["seq"], s["pos"])
