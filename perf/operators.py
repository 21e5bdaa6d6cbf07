"""The performance cases of the operators of a single token's step: matrix-vector products with the packed 4-bit layers,
the norms around a block with its gate and residual scale (forward and backward), and the paged key-value cache with the
attention that reads it.

Kinds of cases (field "kind"):
  matvec   asp_matvec: a packed layer on 1 to 16 unquantized tokens
  norm     block_norm: x' = a x + gate * [norm](branch), h = norm(x') * weight * (1 + scale) + shift
  norm_bwd block_norm_backward: the gradients of x, the branch and every parameter
  attn     paged_attention: one new token per sequence over its pages
  append   kv_append: new keys and values into the pages

Where `own` is false, `run` computes the same in elementary torch operations in 32 bits; where it is true it calls the
package.  Inputs are synthetic: bf16 activations N(0, 1) with 2% of the channels 20 times larger in front of a layer, weights
N(0, 1/K) in the 4-bit group format, caches N(0, 1) whose unwritten slots hold NaN, as memory that nobody wrote can.
"""
import math
import random

import torch

DEV = "cuda"
own = False


def listed():
    return [
        # the action expert's square projection for one token: the smallest call, launch and host path included
        _matvec("matvec_expert_m1", 1, 1024, 1024, r=16),
        # the video transformer's down-projection for a few tokens in the paper's group size, with a bias
        _matvec("matvec_down_m7_g32", 7, 14336, 3072, r=32, group=32, bias=True),
        # a wide 4-bit layer without a branch or smoothing (a language backbone's gate and up projections at once), one token
        _matvec("matvec_plain_m1", 1, 4096, 28672),
        # the norms around one token's block: latency of one row
        _norm("norm_token", 1, 1, 3072, "rms", post=True),
        # a denoising step's rows: LayerNorm with a gate, scale and shift per sample
        _norm("norm_video_t8192", 2, 4096, 3072, "layer", affine=False),
        # probe vectors back through the same rows
        _norm("norm_bwd_t4096", 2, 2048, 3072, "layer", affine=False, bwd=True),
        # post- and pre-norm with learned weights on a float32 residual stream, an odd width
        _norm("norm_bwd_odd_f32", 3, 111, 1001, "rms", post=True, f32=True, bwd=True),
        # the action expert's heads over a short context: latency
        _attn("attn_expert_l77", 1, 16, 1, 64, 77, 16),
        # a batch of ragged contexts, three query heads to a key head, one slot of the batch not in use
        _attn("attn_batch_ragged", 16, 8, 3, 128, 4096, 64),
        # two long contexts in an fp8 cache
        _attn("attn_long_fp8", 2, 8, 3, 128, 131072, 256, fp8=True),
        # one step's keys and values of a batch
        _append("append_step_b16", 16, 1, 8, 128, 64),
        # ragged prompts into an fp8 cache
        _append("append_prompt_fp8", 3, 1365, 8, 128, 32, fp8=True),
    ]


def _matvec(name, M, K, N, r=0, group=64, bias=False):
    return {"name": name, "kind": "matvec", "M": M, "K": K, "N": N, "r": r, "group": group, "bias": bias}


def _norm(name, S, rows, D, norm, post=False, affine=True, f32=False, bwd=False):
    return {"name": name, "kind": "norm_bwd" if bwd else "norm", "S": S, "rows": rows, "D": D, "norm": norm, "post": post,
            "affine": affine, "f32": f32}


def _attn(name, B, H, G, D, L, page, fp8=False, window=0):
    return {"name": name, "kind": "attn", "B": B, "H": H, "G": G, "D": D, "L": L, "page": page, "fp8": fp8, "window": window}


def _append(name, B, L, H, D, page, fp8=False):
    return {"name": name, "kind": "append", "B": B, "L": L, "H": H, "D": D, "page": page, "fp8": fp8}


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _log_step(rng, lo, hi, step):
    return max(lo, min(hi, step * round(_log(rng, lo, hi) / step)))


def draw(rng):
    """One more case of the ranges above: every option of each operator, no case dearer than the largest listed one."""
    kind = rng.choices(["matvec", "norm", "norm_bwd", "attn", "append"], [4, 2, 2, 4, 1])[0]
    if kind == "matvec":
        while True:
            K, N = _log_step(rng, 64, 16384, 64), _log_step(rng, 16, 32768, 16)
            if K * N <= 4096 * 28672:
                break
        c = _matvec("", round(_log(rng, 1, 16)), K, N, r=rng.choice([0, 0, 16, 16, 32, 32, 48, 64]), group=rng.choice([32, 64]),
                    bias=rng.random() < 0.3)
    elif kind in ("norm", "norm_bwd"):
        bwd = kind == "norm_bwd"
        while True:
            S, rows = rng.randint(1, 4), round(_log(rng, 1, 8192))
            D = _log_step(rng, 64, 8192, 8) if rng.random() < 0.7 else round(_log(rng, 33, 4097))
            if S * rows * D <= (4096 if bwd else 8192) * 3072:
                break
        c = _norm("", S, rows, D, rng.choice(["rms", "layer"]), post=rng.random() < 0.5, affine=rng.random() < 0.5,
                  f32=rng.random() < 0.3, bwd=bwd)
    elif kind == "attn":
        while True:
            B, H, D, L = round(_log(rng, 1, 64)), rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 80, 96, 128, 128, 256]), round(_log(rng, 1, 131072))
            if B * H * D * L <= 1024 * 131072:
                break
        c = _attn("", B, H, rng.choice([1, 2, 3, 4, 6, 8, 16, 32]), D, L, rng.choice([16, 32, 64, 128, 256]), fp8=rng.random() < 0.4,
                  window=rng.choice([0, 0, 0, max(1, L // 3)]))
    else:
        while True:
            B, L = round(_log(rng, 1, 64)), round(_log(rng, 1, 4096)) if rng.random() < 0.5 else 1
            if B * L <= 4096:
                break
        c = _append("", B, L, rng.choice([1, 4, 8, 16]), rng.choice([64, 80, 128]), rng.choice([16, 32, 64, 256]), fp8=rng.random() < 0.5)
    del c["name"]
    return c


# ---- inputs, from the seed alone ----

def _gen(seed, salt=0):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 1000003 + salt)


def _quantized(case, seed):
    """Integer codes in [-7, 7] and float32 scales of a random weight: absmax / 7 over each group."""
    M, K, N, gs, r = (case[k] for k in ("M", "K", "N", "group", "r"))
    g = _gen(seed)
    gain = torch.ones(K, device=DEV)
    gain[torch.randperm(K, generator=g, device=DEV)[:max(1, K // 50)]] = 20.0
    x = (torch.randn(M, K, generator=g, device=DEV) * gain).bfloat16()
    inv = (1 / (gain.sqrt() * (0.5 + torch.rand(K, generator=g, device=DEV)))) if r else None     # smoothing goes with the branch
    w = torch.randn(N, K // gs, gs, generator=g, device=DEV) / math.sqrt(K)
    ws = w.abs().amax(dim=2) / 7
    codes = torch.round(w / ws[:, :, None]).clamp_(-7, 7).to(torch.int8).reshape(N, K)
    L1 = (torch.randn(K, r, generator=g, device=DEV) / math.sqrt(K)).bfloat16() if r else None
    L2 = torch.randn(r, N, generator=g, device=DEV).bfloat16() if r else None
    bias = torch.randn(N, generator=g, device=DEV).bfloat16() if case["bias"] else None
    return x, inv, codes, ws, L1, L2, bias


def _pack(codes):
    """Codes int8 [N][K] -> uint8 [N][K/2] in the layers' 8-byte blocks of 16 codes: 6-bit fields sign << 5 | |c| at bits
    6j of a 96-bit stream whose third word sits in the first two words' unused bits."""
    N, K = codes.shape
    c = codes.reshape(N, K // 16, 16).to(torch.int32)
    f = torch.where(c < 0, 32 - c, c).to(torch.int64)
    d = []
    for word in range(3):
        acc = torch.zeros(N, K // 16, dtype=torch.int64, device=codes.device)
        for j in range(16):
            at = 6 * j - 32 * word
            if -6 < at < 32:
                acc |= f[:, :, j] << at if at >= 0 else f[:, :, j] >> -at
        d.append(acc & 0xFFFFFFFF)
    w = (d[0] | (d[2] & 0x18618618)) | ((d[1] | (d[2] & 0x86186186)) << 32)
    return w.contiguous().view(torch.uint8).reshape(N, K // 2)


def _l1_fragments(L1):
    """L1 [K][r] in the activation kernels' fragment order, one of the layer's arrays."""
    K, r = L1.shape
    return L1.reshape(K // 64, 4, 2, 8, r // 16, 16).permute(0, 4, 2, 1, 5, 3).contiguous().reshape(K // 64, r // 16, 2, 64, 8)


def _norm_inputs(case, seed):
    S, rows, D = case["S"], case["rows"], case["D"]
    T, g = S * rows, _gen(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    p = {"x": (2 * rand(T, D) + 0.3).to(torch.float32 if case["f32"] else torch.bfloat16), "branch": rand(T, D).bfloat16(),
         "gate": (0.5 * rand(S, D)).bfloat16(), "scale": (0.3 * rand(S, D)).bfloat16(), "shift": (0.3 * rand(S, D)).bfloat16(),
         "weight": (1 + 0.2 * rand(D)).bfloat16() if case["affine"] else None,
         "post_weight": (1 + 0.2 * rand(D)).bfloat16() if case["post"] and case["affine"] else None}
    if case["kind"] == "norm_bwd":
        p["dxo"], p["dh"] = rand(T, D).to(p["x"].dtype), rand(T, D).bfloat16()
    return p


EPS, RESIDUAL = 1e-5, 0.75


def _lengths(case):
    """Ragged context lengths of a batch, the same for every seed: the longest first, the second slot of four or more unused."""
    B, L = case["B"], case["L"]
    r = random.Random(B * 1000003 + L)
    n = [L] + [max(1, round(_log(r, max(1, L / 32), L))) for _ in range(B - 1)]
    if B >= 4:
        n[1] = 0
    return n


def _cache(case, lengths, g, extra=0):
    """Pages of random values in a shuffled order, tables whose unused entries are -1, and NaN in every slot past a length."""
    B, H, D, P = case["B"], case["H"], case["D"], case["page"]
    used = [-(-(n + extra) // P) for n in lengths]
    width, total = max(1, max(used)), sum(used) + 1
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    shape, kind = (total, H, P, D), torch.float8_e4m3fn if case["fp8"] else torch.bfloat16
    written = torch.zeros(total, P, dtype=torch.bool, device=DEV)
    at = 0
    for b, n in enumerate(lengths):
        table[b, :used[b]] = order[at:at + used[b]]
        full = torch.arange(used[b] * P, device=DEV).reshape(-1, P) < n
        written[order[at:at + used[b]].long()] = full
        at += used[b]
    out = []
    for _ in range(2):
        c = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        c = torch.where(written[:, None, :, None], c, torch.full((), float("nan"), dtype=torch.bfloat16, device=DEV))
        out.append((c * 64).to(kind) if case["fp8"] else c)
        del c
    scales = (torch.exp2(torch.randint(-7, -4, (H,), generator=g, device=DEV).float()) if case["fp8"] else None for _ in range(2))
    return (*out, table, *scales)


def prepare(case, seed):
    k = case["kind"]
    if k == "matvec":
        x, inv, codes, ws, L1, L2, bias = _quantized(case, seed)
        layer = {"K": case["K"], "N": case["N"], "r": case["r"], "group": case["group"], "wq": _pack(codes), "ws": ws.t().contiguous(),
                 "inv_smooth": inv, "bias": bias, "L1t": None, "L2t": None}
        if case["r"]:
            layer.update(L1t=L1.t().contiguous(), L2t=L2.t().contiguous(), L1f=_l1_fragments(L1))
        return {"kind": k, "x": x, "layer": layer}
    if k in ("norm", "norm_bwd"):
        return {"kind": k, "norm": case["norm"], "post": case["post"], **_norm_inputs(case, seed)}
    g = _gen(seed)
    if k == "attn":
        n = _lengths(case)
        K, V, table, ks, vs = _cache(case, n, g)
        q = torch.randn(case["B"], case["H"] * case["G"], case["D"], generator=g, device=DEV).bfloat16()
        lengths = torch.tensor(n, dtype=torch.int32, device=DEV)
        starts = torch.clamp(lengths - case["window"], min=0) if case["window"] else None
        return {"kind": k, "q": q, "cache": (K, V, table, ks, vs), "lengths": lengths, "starts": starts, "scale": case["D"] ** -0.5}
    # a step appends one token to each ragged context; a prompt fills an empty cache
    B, L, H, D = (case[f] for f in ("B", "L", "H", "D"))
    if L == 1:
        before, new = [37 * b % 512 for b in range(B)], [1] * B
    else:
        new = _lengths(case)
        before = [0] * B
    K, V, table, ks, vs = _cache({**case, "fp8": case["fp8"]}, [a + n for a, n in zip(before, new)], g)
    for c in (K, V):
        c.copy_(torch.zeros((), dtype=torch.bfloat16, device=DEV).to(c.dtype).expand_as(c))
    T = sum(new)
    kv = torch.randn(2, T, H, D, generator=g, device=DEV).bfloat16()
    seq = torch.tensor([b for b, n in enumerate(new) for _ in range(n)], dtype=torch.int32, device=DEV)
    pos = torch.tensor([a + i for a, n in zip(before, new) for i in range(n)], dtype=torch.int32, device=DEV)
    return {"kind": k, "k": kv[0], "v": kv[1], "cache": (K, V, table, ks, vs), "seq": seq, "pos": pos}


# ---- one pass ----

def _own_run(s):
    import paper_2609_33269_amd as qwam
    k = s["kind"]
    if k == "matvec":
        if "handle" not in s:          # the layer object that a program holds beside its arrays
            s["handle"] = qwam.PackedLayer(**s["layer"])
        return qwam.asp_matvec(s["handle"], s["x"])
    if k == "norm":
        return qwam.block_norm(s["x"], s["branch"], norm=s["norm"], eps=EPS, residual_scale=RESIDUAL, gate=s["gate"], post_norm=s["post"],
                               post_weight=s["post_weight"], weight=s["weight"], scale=s["scale"], shift=s["shift"])
    if k == "norm_bwd":
        return qwam.block_norm_backward(s["dxo"], s["dh"], s["x"], s["branch"], norm=s["norm"], eps=EPS, residual_scale=RESIDUAL,
                                        gate=s["gate"], post_norm=s["post"], post_weight=s["post_weight"], weight=s["weight"],
                                        scale=s["scale"], shift=s["shift"])
    if "handle" not in s:
        s["handle"] = qwam.PagedCache(*s["cache"])
    if k == "attn":
        return qwam.paged_attention(s["handle"], s["q"], s["lengths"], starts=s["starts"], scale=s["scale"])
    qwam.kv_append(s["handle"], s["k"], s["v"], s["seq"], s["pos"])
    return s["cache"][:2]


def run(s):
    if own:
        return _own_run(s)
    k = s["kind"]
    if k == "matvec":
        return _plain_matvec(s["layer"], s["x"])
    if k == "norm":
        return _plain_norm(s)
    if k == "norm_bwd":
        return _plain_norm_bwd(s)
    if k == "attn":
        return _plain_attn(s)
    return _plain_append(s)


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ----

def _plain_matvec(p, x):
    w = p["wq"].view(torch.int64)                                       # [N][K/16], one code block each
    lo, hi = w & 0xFFFFFFFF, (w >> 32) & 0xFFFFFFFF
    d2 = (lo & 0x18618618) | (hi & 0x86186186)
    d01 = (lo & 0xE79E79E7) | ((hi & 0x79E79E79) << 32)                 # stream bits 0..63
    d12 = (d01 >> 60 & 0xF) | (d2 << 4)                                 # stream bits 60..95
    at = torch.arange(0, 60, 6, device=w.device)
    f = torch.cat(((d01[:, :, None] >> at) & 63, (d12[:, :, None] >> at[:6]) & 63), dim=2).to(torch.int32)
    c = torch.where(f >= 32, 32 - f, f).to(torch.float32)
    c = (c.reshape(p["N"], -1, p["group"]) * p["ws"].t()[:, :, None]).reshape(p["N"], p["K"])
    xt = x.float()
    if p["inv_smooth"] is not None:
        xt = xt * p["inv_smooth"]
    y = xt @ c.t()
    if p["r"]:
        y = y + (xt @ p["L1t"].float().t()) @ p["L2t"].float().t()
    if p["bias"] is not None:
        y = y + p["bias"].float()
    return y.bfloat16()


def _f(t):
    return None if t is None else t.float()


def _unit(v, norm):
    """v normalized over its last axis, and 1 / its deviation."""
    if norm == "layer":
        v = v - v.mean(-1, keepdim=True)
    r = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * r, r


def _plain_norm(s):
    S, (T, D) = s["gate"].shape[0], s["x"].shape
    u = s["branch"].float()
    if s["post"]:
        u = _unit(u, s["norm"])[0]
        if s["post_weight"] is not None:
            u = u * s["post_weight"].float()
    xo = RESIDUAL * s["x"].float().reshape(S, -1, D) + s["gate"].float()[:, None] * u.reshape(S, -1, D)
    h = _unit(xo, s["norm"])[0]
    if s["weight"] is not None:
        h = h * s["weight"].float()
    h = h * (1 + s["scale"].float()[:, None]) + s["shift"].float()[:, None]
    return xo.reshape(T, D).to(s["x"].dtype), h.reshape(T, D).bfloat16()


def _unit_grad(e, z, r, norm):
    """The gradient of v where e is that of z = unit(v)."""
    e = e - z * (e * z).mean(-1, keepdim=True)
    if norm == "layer":
        e = e - e.mean(-1, keepdim=True)
    return e * r


def _plain_norm_bwd(s):
    S, (T, D) = s["gate"].shape[0], s["x"].shape
    of = lambda n: s[n].float().reshape(S, -1, D)  # noqa: E731
    dh, gate, wp = of("dh"), s["gate"].float()[:, None], _f(s["post_weight"])
    z, r = _unit(of("x"), s["norm"])
    w = _f(s["weight"])
    f = 1 + s["scale"].float()[:, None]
    if w is not None:
        f = f * w
    d = of("dxo") + _unit_grad(dh * f, z, r, s["norm"])
    u, e = of("branch"), gate * d
    if s["post"]:
        u, rb = _unit(u, s["norm"])
        db = _unit_grad(e if wp is None else e * wp, u, rb, s["norm"])
    else:
        db = e
    a, c = (dh * z).sum(1), (d * u).sum(1)
    return {"dx": (RESIDUAL * d).reshape(T, D).to(s["x"].dtype), "dbranch": db.reshape(T, D).bfloat16(), "dgate": c if wp is None else c * wp,
            "dpost_weight": None if wp is None else (c * gate[:, 0]).sum(0), "dweight": None if w is None else (a * (1 + s["scale"].float())).sum(0),
            "dscale": a if w is None else a * w, "dshift": dh.sum(1)}


def _plain_attn(s):
    K, V, table, ks, vs = s["cache"]
    q, n = s["q"].float(), s["lengths"]
    (B, Hq, D), (_, H, P, _) = q.shape, K.shape
    at = torch.arange(table.shape[1] * P, device=q.device)
    seen = at[None] < n[:, None]
    if s["starts"] is not None:
        seen = seen & (at[None] >= s["starts"][:, None])
    idx = table.clamp(min=0).long()
    view = lambda c: c.view(torch.uint8)[idx].view(c.dtype) if c.dtype == torch.float8_e4m3fn else c[idx]  # noqa: E731
    k = view(K).float().transpose(1, 2).reshape(B, H, -1, D)
    v = view(V).float().transpose(1, 2).reshape(B, H, -1, D)
    k = torch.where(seen[:, None, :, None], k, 0.0)
    v = torch.where(seen[:, None, :, None], v, 0.0)
    if ks is not None:
        k, v = k * ks[:, None, None], v * vs[:, None, None]
    x = (q.reshape(B, H, -1, D) * s["scale"]) @ k.transpose(2, 3)
    x = torch.where(seen[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    o = (e @ v) / e.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.reshape(B, Hq, D).bfloat16()


def _plain_append(s):
    K, V, table, ks, vs = s["cache"]
    P = K.shape[2]
    seq, pos = s["seq"].long(), s["pos"].long()
    page = table[seq, pos // P].long()
    for c, x, scale in ((K, s["k"], ks), (V, s["v"], vs)):
        if scale is not None:
            x = (x.float() / scale[:, None]).clamp(-448, 448).to(c.dtype)
            c, x = c.view(torch.uint8), x.view(torch.uint8)
        c[page, :, pos % P] = x
    return K, V


# ---- what one pass cannot do without ----

def work(case):
    k = case["kind"]
    if k == "matvec":
        M, K, N, r, g = (case[f] for f in ("M", "K", "N", "r", "group"))
        b = N * K // 2 + 4 * N * (K // g) + 2 * M * K + 2 * M * N + (4 * K + 2 * r * (K + N) if r else 0) + (2 * N if case["bias"] else 0)
        return {"bytes": b, "flops": 2 * M * K * N + 2 * M * r * (K + N)}
    if k in ("norm", "norm_bwd"):
        T, D, e = case["S"] * case["rows"], case["D"], 4 if case["f32"] else 2
        par = 6 * case["S"] * D + 2 * D * (case["affine"] + (case["affine"] and case["post"]))
        if k == "norm":
            return {"bytes": T * D * (2 * e + 4) + par, "flops": 12 * T * D}
        return {"bytes": T * D * (3 * e + 6) + 3 * par, "flops": 25 * T * D}
    e = 1 if case["fp8"] else 2
    if k == "attn":
        B, H, G, D = (case[f] for f in ("B", "H", "G", "D"))
        seen = sum(min(n, case["window"] or n) for n in _lengths(case))
        return {"bytes": 2 * seen * H * D * e + 4 * B * H * G * D + 4 * sum(-(-n // case["page"]) for n in _lengths(case)),
                "flops": 4 * seen * H * G * D}
    T = case["B"] if case["L"] == 1 else sum(_lengths(case))
    return {"bytes": 2 * T * case["H"] * case["D"] * (2 + e) + 8 * T, "flops": 0}


# ---- the same in 64 bits, from the definitions ----

def _exact_matvec(case, seed):
    x, inv, codes, ws, L1, L2, bias = _quantized(case, seed)
    x = x.double() if inv is None else x.double() * inv.double()
    G = case["K"] // case["group"]
    y = torch.zeros(case["M"], case["N"], dtype=torch.float64, device=DEV)
    for g in range(G):                                               # one group of channels at a time
        at = slice(g * case["group"], (g + 1) * case["group"])
        y += (x[:, at] @ codes[:, at].double().t().contiguous()) * ws[:, g].double()
    if L1 is not None:
        y += x @ (L1.double() @ L2.double()) if case["N"] * case["K"] < 1 << 27 else (x @ L1.double()) @ L2.double()
    return y if bias is None else y + bias.double()


def _exact_rows(case, seed):
    """Row by row of samples, with autograd for the backward pass."""
    p = _norm_inputs(case, seed)
    bwd = case["kind"] == "norm_bwd"
    leaf = {n: t.double().requires_grad_(bwd) for n, t in p.items() if t is not None and n not in ("dxo", "dh")}
    T, D = leaf["x"].shape
    row = torch.arange(T, device=DEV) // case["rows"]

    def normal(v):
        m = v.mean(dim=1, keepdim=True) if case["norm"] == "layer" else 0
        return (v - m) / torch.sqrt(((v - m) ** 2).sum(dim=1, keepdim=True) / D + EPS)

    b = normal(leaf["branch"]) if case["post"] else leaf["branch"]
    b = b * leaf.get("post_weight", 1)
    kept = b * leaf["gate"][row]
    # backward is taken at the stored sum, so x stands for it there and the branch's share cancels in value only
    xo = leaf["x"] + (kept - kept.detach()) if bwd else RESIDUAL * leaf["x"] + kept
    h = normal(xo) * leaf.get("weight", 1) * (1 + leaf["scale"][row]) + leaf["shift"][row]
    if not bwd:
        return xo, h
    torch.autograd.backward([xo, h], [p["dxo"].double(), p["dh"].double()])
    grad = lambda n: leaf[n].grad if n in leaf else None  # noqa: E731
    return {"dx": RESIDUAL * leaf["x"].grad, "dbranch": grad("branch"), "dgate": grad("gate"), "dpost_weight": grad("post_weight"),
            "dweight": grad("weight"), "dscale": grad("scale"), "dshift": grad("shift")}


def _exact_attn(case, seed):
    s = prepare(case, seed)
    K, V, table, ks, vs = s["cache"]
    H, G, D = case["H"], case["G"], case["D"]
    out = torch.zeros(case["B"], H * G, D, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(case)):
        first = max(0, n - case["window"]) if case["window"] else 0
        if first >= n:
            continue
        pages = table[b, :-(-n // case["page"])].tolist()
        for h in range(H):
            k, v = (torch.cat([c[p, h].double() for p in pages])[first:n] for c in (K, V))
            if ks is not None:
                k, v = k * ks[h].double(), v * vs[h].double()
            w = torch.softmax(s["q"][b, h * G:(h + 1) * G].double() @ k.t().contiguous() * case["D"] ** -0.5, dim=-1)
            out[b, h * G:(h + 1) * G] = w @ v
    return out


def exact(case, seed):
    k = case["kind"]
    if k == "matvec":
        return _exact_matvec(case, seed)
    if k in ("norm", "norm_bwd"):
        return _exact_rows(case, seed)
    if k == "attn":
        return _exact_attn(case, seed) if case["B"] * case["H"] * case["L"] // case["page"] < 300000 else None
    return None                # stored values, not computed ones
