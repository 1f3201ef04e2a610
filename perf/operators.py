"""The 8-bit KV cache, paged attention and packed attention: the calls that are timed,
their plain forms, and the sizes users run.

A case is one pass of one kind:

  kv8     one iteration's part of a layer whose KV cache is kept in 8 bits: the fresh
          rows of the active tokens are quantised into it (K rotated on its way, or
          not), then the whole layer is read back for the attention over it.
  paged   a few new tokens per sequence against caches held in pages, bf16 or 8-bit:
          sequences of their own lengths, query heads in groups that share a K/V head.
  packed  several sequences packed one behind the other, all their queries at once:
          bidirectional (mask 0), causal (mask 1), or causal by frames of `mask`
          tokens; a sequence may continue one whose first keys are older.

With `own` the calls of this library run; without it the same results come from
elementary torch operations in 32 bits, rounded once.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # A small fp32 layer (4x16x16 tokens, 4 heads x 64), a quarter of the tokens
        # active: the smallest use, all launch latency.
        {"name": "kv8_tiny_f32", "kind": "kv8", "F": 4, "Hh": 16, "Ww": 16, "H": 4, "D": 64,
         "dtype": "f32", "share": 0.25, "rope": False},
        # An LTX-like layer (16x16x24 tokens, 32 heads x 64), three quarters of the
        # tokens active, K rotated on its way: the ordinary iteration.
        {"name": "kv8_ltx_most", "kind": "kv8", "F": 16, "Hh": 16, "Ww": 24, "H": 32, "D": 64,
         "dtype": "bf16", "share": 0.75, "rope": True},
        # A Wan-14B-like layer (40 heads x 128) of a 720p-like video (21x45x80 tokens),
        # a quarter of the tokens active: the largest.
        {"name": "kv8_720p_quarter", "kind": "kv8", "F": 21, "Hh": 45, "Ww": 80, "H": 40,
         "D": 128, "dtype": "bf16", "share": 0.25, "rope": True},
        # One new token of one sequence of 4001: the latency of a single user's step.
        {"name": "token_one", "kind": "paged", "batch": 1, "lo": 4001, "hi": 4001, "mix": 1,
         "new": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 16, "cache": "bf16"},
        # One new token of 48 sequences of mixed ages in an 8-bit cache: a busy server.
        {"name": "token_ragged_e4m3", "kind": "paged", "batch": 48, "lo": 100, "hi": 9000,
         "mix": 2, "new": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "cache": "e4m3"},
        # Four sequences of up to 128k tokens: few rows, long caches.
        {"name": "token_long", "kind": "paged", "batch": 4, "lo": 60000, "hi": 131072, "mix": 3,
         "new": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 128, "cache": "bf16"},
        # Four drafted tokens per sequence, each head with its own K/V (12 heads x 64).
        {"name": "draft4_mha_e4m3", "kind": "paged", "batch": 16, "lo": 300, "hi": 12000,
         "mix": 4, "new": 4, "Hq": 12, "Hkv": 12, "D": 64, "page": 32, "cache": "e4m3"},
        # Three short sequences without a mask (conditioning tokens): the smallest call.
        {"name": "packed_short", "kind": "packed", "batch": 3, "lo": 1, "hi": 190, "mix": 5,
         "older": 0, "Hq": 8, "Hkv": 2, "D": 64, "mask": 0},
        # Six prompts of 500 to 6000 tokens, causal: the ordinary prompt batch.
        {"name": "packed_prompts", "kind": "packed", "batch": 6, "lo": 500, "hi": 6000, "mix": 6,
         "older": 0, "Hq": 32, "Hkv": 8, "D": 128, "mask": 1},
        # Two LTX-like videos (16 frames of 384 tokens, 32 heads x 64), causal by frames.
        {"name": "packed_frames_ltx", "kind": "packed", "batch": 2, "lo": 6144, "hi": 6144,
         "mix": 7, "older": 0, "Hq": 32, "Hkv": 32, "D": 64, "mask": 384},
        # Two prompts continued by 512 tokens each after 9000 to 20000 older ones: few
        # rows, long keys.
        {"name": "packed_continued", "kind": "packed", "batch": 2, "lo": 512, "hi": 512,
         "mix": 8, "older": 20000, "Hq": 16, "Hkv": 2, "D": 128, "mask": 1},
        # One prompt of 16384 tokens: the largest call.
        {"name": "packed_long", "kind": "packed", "batch": 1, "lo": 16384, "hi": 16384, "mix": 9,
         "older": 0, "Hq": 16, "Hkv": 2, "D": 128, "mask": 1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["kv8", "paged", "packed"])
    if kind == "kv8":
        H, D = rng.choice([1, 3, 4, 7, 12, 24, 32, 40]), rng.choice([32, 64, 64, 96, 128, 128])
        n = _log(rng, 300, min(75600, 387_000_000 // (H * D)))
        Hh, Ww = rng.randint(1, 17), rng.randint(1, 17)
        rope = rng.random() < 0.6
        return {"kind": kind, "F": max(1, n // (Hh * Ww)), "Hh": Hh, "Ww": Ww, "H": H, "D": D,
                "dtype": "bf16" if rope or rng.random() < 0.6 else "f32",
                "share": round(rng.uniform(0.05, 1.0), 3), "rope": rope}
    D = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
    if kind == "paged":
        hi = _log(rng, 64, 131072)
        batch = _log(rng, 1, max(1.0, min(96.0, 260000.0 * 8 / (hi * Hkv))))
        return {"kind": kind, "batch": batch, "lo": max(1, int(hi * rng.choice([0.02, 0.3, 1.0]))),
                "hi": hi, "mix": rng.randrange(1 << 30), "new": rng.choice([1, 1, 1, 2, 3, 5]),
                "Hq": Hq, "Hkv": Hkv, "D": D, "page": rng.choice([8, 16, 32, 64, 128, 256]),
                "cache": rng.choice(["bf16", "e4m3"])}
    Hq = min(Hq, 32) // Hkv * Hkv
    pairs = 16384 * 16384 * 16 * 128 // (2 * Hq * D)   # the largest listed case's work
    hi = min(_log(rng, 16, min(12000.0, math.sqrt(pairs))), math.isqrt(pairs))
    batch = min(_log(rng, 1, max(1.0, min(24.0, pairs / hi ** 2))), max(1, pairs // hi ** 2))
    older = rng.choice([0, 0, rng.randint(0, max(0, min(20000, pairs // (batch * hi) - hi)))])
    return {"kind": kind, "batch": batch, "lo": max(1, int(hi * rng.choice([0.05, 0.4, 1.0]))),
            "hi": hi, "mix": rng.randrange(1 << 30), "older": older, "Hq": Hq, "Hkv": Hkv, "D": D,
            "mask": rng.choice([0, 1, 1, rng.randint(2, 500)])}


# ------------------------------------------------------------------ sizes

def _lengths(case):
    """(query, key) length of each sequence."""
    r = random.Random(case["mix"])
    out = []
    for _ in range(case["batch"]):
        q = r.randint(case["lo"], case["hi"])
        older = case.get("older", 0)
        out.append((q, q + (r.randint(int(older * 0.45), older) if older else 0)))
    return out


def _limits(lq, lk, mask):
    """Number of keys that each of lq queries may see."""
    if not mask:
        return [lk] * lq
    return [min(lk, ((i + lk - lq) // mask + 1) * mask) for i in range(lq)]


def work(case):
    if case["kind"] == "kv8":
        n_all = case["F"] * case["Hh"] * case["Ww"]
        n = max(1, int(n_all * case["share"]))
        H, D, w = case["H"], case["D"], 2 if case["dtype"] == "bf16" else 4
        write = n * (2 * H * D * w + 2 * H * (D + 1) + 4 + (4 * D if case["rope"] else 0))
        read = n_all * (2 * H * (D + 1) + 2 * H * D * w)
        return {"bytes": write + read, "flops": (8 if case["rope"] else 4) * n * H * D}
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    lens = _lengths(case)
    if case["kind"] == "paged":
        new, w = case["new"], 2 * D if case["cache"] == "bf16" else D + 1
        keys = sum(k for _, k in lens)
        pairs = sum(max(0, k - new + i + 1) for _, k in lens for i in range(new))
        return {"bytes": 2 * keys * Hkv * w + 2 * case["batch"] * new * Hq * D * 2 +
                4 * sum(-(-k // case["page"]) for _, k in lens), "flops": 4 * D * Hq * pairs}
    pairs = sum(sum(max(0, x) for x in _limits(q, k, case["mask"])) for q, k in lens)
    return {"bytes": 2 * D * (2 * Hq * sum(q for q, _ in lens) + 2 * Hkv * sum(k for _, k in lens)),
            "flops": 4 * D * Hq * pairs}


# ----------------------------------------------------------------- inputs

def _normal(g, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _keys(g, rows, H, D, dtype=torch.bfloat16):
    """Keys have a few channels that are larger than the others, as trained models' do."""
    k = torch.randn((rows, H, D), generator=g, device=DEV, dtype=torch.float32)
    big = torch.rand((1, H, D), generator=g, device=DEV) < 0.03
    return (k * torch.where(big, 4.0, 0.9)).to(dtype)


def _power(e):
    """2^e in 32 bits, e an integer tensor in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x):
    """(e4m3 codes, exponents) of the rows x[..., D], in 32 bits: the least power of two
    that brings a row's largest value to 448 or less, at least 2^-100."""
    x = x.float().clamp(-1.875 * 2.0 ** 127, 1.875 * 2.0 ** 127)
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(m == 0, torch.full_like(e, -100), e).clamp(min=-100)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn), e


def _values(code, e):
    return code.float() * _power(e)[..., None]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 17)
    D = case["D"]
    s = {"case": case}
    if case["kind"] == "kv8":
        dt, H = DTYPES[case["dtype"]], case["H"]
        N = case["F"] * case["Hh"] * case["Ww"]
        n = max(1, int(N * case["share"]))
        s["idx"] = torch.randperm(N, generator=g, device=DEV)[:n].sort().values.int()
        s["k_fresh"], s["v_fresh"] = _keys(g, n, H, D, dt), _normal(g, (n, H, D), dt)
        # the layer's cache as the iterations before left it
        for name, x in (("k", _keys(g, N, H, D)), ("v", _normal(g, (N, H, D)))):
            code, e = _quantise(x)
            s[name + "_cache"], s[name + "_scale"] = code, (e + 127).to(torch.uint8)
            s[name + "_out"] = torch.empty((N, H, D), dtype=dt, device=DEV)
        s["table"] = None
        if case["rope"]:
            # angles of far positions need 64 bits
            band = [D // 2 - 2 * (D // 6), D // 6, D // 6]
            at = torch.arange(N, device=DEV)
            axes = (at // (case["Hh"] * case["Ww"]), at // case["Ww"] % case["Hh"],
                    at % case["Ww"])
            a = torch.cat([p[:, None].double() *
                           10000.0 ** (-torch.arange(b, device=DEV).double() / max(b, 1))
                           for p, b in zip(axes, band)], 1)
            s["table"] = torch.stack([a.cos(), a.sin()], -1).float()
        return s
    Hq, Hkv = case["Hq"], case["Hkv"]
    s["lens"] = _lengths(case)
    if case["kind"] == "paged":
        P, B = case["page"], case["batch"]
        need = [-(-k // P) for _, k in s["lens"]]
        pages = sum(need) + 3
        ids = torch.randperm(pages, generator=g, device=DEV).int()
        s["table"] = torch.zeros((B, max(need)), dtype=torch.int32, device=DEV)
        at = 0
        for b, c in enumerate(need):
            s["table"][b, :c] = ids[at:at + c]
            at += c
        s["seq_lens"] = torch.tensor([k for _, k in s["lens"]], dtype=torch.int32, device=DEV)
        s["q"] = _normal(g, (B, case["new"], Hq, D))
        for name, make in (("k", _keys), ("v", lambda g, r, h, d: _normal(g, (r, h, d)))):
            x = make(g, pages * P, Hkv, D).view(pages, P, Hkv, D)
            s[name + "_scale"] = None
            if case["cache"] == "e4m3":
                x, e = _quantise(x)
                s[name + "_scale"] = (e + 127).to(torch.uint8)
            s[name + "_pages"] = x
        s["out"] = torch.empty_like(s["q"])
        s["workspace"] = None
        return s
    cum = [0], [0]
    for q, k in s["lens"]:
        cum[0].append(cum[0][-1] + q)
        cum[1].append(cum[1][-1] + k)
    s["cu_q"], s["cu_k"] = (torch.tensor(c, dtype=torch.int32, device=DEV) for c in cum)
    s["q"] = _normal(g, (cum[0][-1], Hq, D))
    s["k"], s["v"] = _keys(g, cum[1][-1], Hkv, D), _normal(g, (cum[1][-1], Hkv, D))
    s["out"] = torch.empty_like(s["q"])
    s["workspace"] = None
    return s


# -------------------------------------------------------------------- run

def run(s):
    if own:
        return _run_own(s)
    return {"kv8": _kv8, "paged": _paged, "packed": _packed}[s["case"]["kind"]](s)


def _run_own(s):
    import paper_2605_06892_gb300 as hsa
    kind = s["case"]["kind"]
    if kind == "kv8":
        n, N = s["idx"].numel(), s["k_cache"].shape[0]
        hsa.hsa_kv_quant_scatter(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                                 s["k_fresh"], s["v_fresh"], s["idx"], n, table=s["table"])
        hsa.hsa_kv_dequant_gather(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], None, N,
                                  s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"], "k_scale": s["k_scale"],
                "v_scale": s["v_scale"]}
    if s["workspace"] is None:   # once, kept as a user's program keeps it
        c = s["case"]
        size = (hsa.hsa_paged_attention_workspace_bytes(c["batch"], c["new"], c["Hq"], c["Hkv"],
                                                        c["D"])
                if kind == "paged" else
                hsa.hsa_packed_attention_workspace_bytes(c["Hq"], c["Hkv"], c["D"]))
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    if kind == "paged":
        hsa.hsa_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["seq_lens"],
                                s["out"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                workspace=s["workspace"])
    else:
        hsa.hsa_packed_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["out"],
                                 mask=s["case"]["mask"], workspace=s["workspace"])
    return s["out"]


def _kv8(s):
    idx = s["idx"].long()
    k = s["k_fresh"]
    if s["table"] is not None:
        # the rotation rounds to 32 bits after each step and then to bf16, as that of the
        # bf16 cache does; 64 bits hold the products, so that no border is missed
        x0, x1 = (x.double() for x in k.unflatten(-1, (-1, 2)).unbind(-1))
        c, sn = (x.double() for x in s["table"][idx][:, None].unbind(-1))
        y0 = (x0 * c - (x1 * sn).float().double()).float()
        y1 = (x0 * sn + (x1 * c).float().double()).float()
        k = torch.stack([y0, y1], -1).flatten(-2).to(k.dtype)
    out = {}
    for name, x in (("k", k), ("v", s["v_fresh"])):
        code, e = _quantise(x)
        # indexed writes of 8-bit floats go by their bits
        s[name + "_cache"].view(torch.uint8)[idx] = code.view(torch.uint8)
        s[name + "_scale"][idx] = (e + 127).to(torch.uint8)
        out[name] = _values(s[name + "_cache"], s[name + "_scale"].int() - 127).to(
            s[name + "_out"].dtype)
        out[name + "_scale"] = s[name + "_scale"]
    return out


def _attend(q, k, v, limit):
    """Queries [n, Hkv, G, D] against k, v [m, Hkv, D]; query i sees the first limit[i]."""
    n, Hkv, G, D = q.shape
    q, k, v = q.permute(1, 0, 2, 3).float(), k.transpose(0, 1).float(), v.transpose(0, 1).float()
    x = torch.matmul(q.reshape(Hkv, n * G, D), k.transpose(1, 2)) / math.sqrt(D)
    seen = torch.arange(k.shape[1], device=DEV) < limit.repeat_interleave(G)[:, None]
    x = x.masked_fill_(~seen, -math.inf)
    x = torch.exp(x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)))
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.view(Hkv, n, G, D).permute(1, 0, 2, 3)


def _limit(lq, lk, mask):
    p = torch.arange(lq, device=DEV) + (lk - lq)
    return torch.full_like(p, lk) if not mask else ((p // mask + 1) * mask).clamp(max=lk)


def _rows(s, b):
    """Keys and values [len, Hkv, D] of one sequence of the paged cache, in 32 bits."""
    c = s["case"]
    n = s["lens"][b][1]
    ids = s["table"][b, :-(-n // c["page"])].long()
    out = []
    for name in ("k", "v"):
        x = s[name + "_pages"][ids] if c["cache"] == "bf16" else _values(
            s[name + "_pages"].view(torch.uint8)[ids].view(torch.float8_e4m3fn),
            s[name + "_scale"][ids].int() - 127)
        out.append(x.flatten(0, 1)[:n].float())
    return out


def _paged(s):
    c = s["case"]
    q = s["q"].unflatten(2, (c["Hkv"], -1))
    return torch.stack([_attend(q[b], *_rows(s, b), _limit(c["new"], n, 1)).flatten(1, 2)
                        for b, (_, n) in enumerate(s["lens"])]).to(s["q"].dtype)


def _packed(s):
    c = s["case"]
    q = s["q"].unflatten(1, (c["Hkv"], -1))
    out = torch.empty_like(q)
    q0 = k0 = 0
    for lq, lk in s["lens"]:
        limit = _limit(lq, lk, c["mask"])
        for h in range(c["Hkv"]):   # a K/V head at a time bounds the memory
            at = (slice(k0, k0 + lk), slice(h, h + 1))
            out[q0:q0 + lq, h:h + 1] = _attend(q[q0:q0 + lq, h:h + 1], s["k"][at], s["v"][at],
                                               limit).to(out.dtype)
        q0, k0 = q0 + lq, k0 + lk
    return out.flatten(1, 2)


# ------------------------------------------------------------------ exact

def _rounded(x, bits, least):
    """64-bit values to `bits` significant bits, ties to even; steps of 2^least at least."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - bits).clamp(min=least).double())
    return torch.round(x / step) * step


def _exact_rows(x):
    """Values and exponents that the 8-bit cache holds for the 64-bit rows x."""
    x = x.clamp(-1.875 * 2.0 ** 127, 1.875 * 2.0 ** 127)
    a = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 448.0))
    e = torch.where(a * torch.exp2(-e) > 448.0, e + 1, e)     # the logarithm's own rounding
    e = torch.where(a * torch.exp2(1 - e) <= 448.0, e - 1, e).clamp(min=-100.0)
    return _rounded(x * torch.exp2(-e), 4, -9) * torch.exp2(e), e[..., 0]


def _exact_attention(q, k, v, first, mask):
    """Rows q [n, Hq, D] of positions first, first + 1, ... against k, v [m, Hkv, D]."""
    n, Hq, D = q.shape
    m, G = k.shape[0], Hq // k.shape[1]
    out = torch.zeros((n, Hq, D), dtype=torch.float64, device=DEV)
    key = torch.arange(m, device=DEV)
    for r0 in range(0, n, 2048):
        p = torch.arange(r0, min(n, r0 + 2048), device=DEV) + first
        hide = torch.zeros((p.numel(), m), dtype=torch.bool, device=DEV)
        if mask:
            hide = torch.div(key, mask, rounding_mode="floor") > torch.div(
                p, mask, rounding_mode="floor")[:, None]
        for h in range(Hq):
            x = q[r0:r0 + 2048, h].double() @ k[:, h // G].double().t() * D ** -0.5
            w = torch.softmax(x.masked_fill(hide, -math.inf), -1)
            out[r0:r0 + 2048, h] = torch.where(hide.all(-1, keepdim=True), 0.0,
                                               w @ v[:, h // G].double())
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "kv8":
        idx, out = s["idx"].long(), {}
        k = s["k_fresh"].double()
        if s["table"] is not None:
            a, b = k[..., 0::2], k[..., 1::2]
            c, sn = (s["table"][idx, :, i].double()[:, None] for i in (0, 1))
            k = torch.empty_like(k)
            k[..., 0::2] = a * c - _rounded(b * sn, 24, -149)
            k[..., 1::2] = a * sn + _rounded(b * c, 24, -149)
            k = _rounded(_rounded(k, 24, -149), 8, -133)
        for name, x in (("k", k), ("v", s["v_fresh"].double())):
            e_all = s[name + "_scale"].double() - 127
            all_rows = s[name + "_cache"].double() * torch.exp2(e_all)[..., None]
            all_rows[idx], e_all[idx] = _exact_rows(x)
            out[name], out[name + "_scale"] = all_rows, (e_all + 127).to(torch.uint8)
        return out
    lens = s["lens"]
    if case["kind"] == "paged":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        for b, (_, n) in enumerate(lens):
            at = torch.arange(n, device=DEV)
            page, row = s["table"][b, at // case["page"]].long(), at % case["page"]
            kv = []
            for name in ("k", "v"):
                x = s[name + "_pages"]
                x = (x.view(torch.uint8)[page, row].view(torch.float8_e4m3fn).double()
                     if case["cache"] == "e4m3" else x[page, row].double())
                if case["cache"] == "e4m3":
                    x = x * torch.exp2(s[name + "_scale"][page, row].double() - 127)[..., None]
                kv.append(x)
            out[b] = _exact_attention(s["q"][b], kv[0], kv[1], n - case["new"], 1)
        return out
    out, q0, k0 = [], 0, 0
    for lq, lk in lens:
        out.append(_exact_attention(s["q"][q0:q0 + lq], s["k"][k0:k0 + lk], s["v"][k0:k0 + lk],
                                    lk - lq, case["mask"]))
        q0, k0 = q0 + lq, k0 + lk
    return torch.cat(out)
