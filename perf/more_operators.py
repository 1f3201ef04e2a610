"""Page planning, normed and rotated queries and keys, the 4-bit KV cache and attention over
it: the calls that are timed, their plain forms, and the sizes users run.

A case is one pass of one kind:

  plan    the bookkeeping before a server's step: from each sequence's present and wanted
          length the pages it takes or gives back, the rows of the cache that its new
          tokens go to, their positions, and the offsets of the packed batch; with `keys`
          also the cache rows of all its keys.
  norm    the queries and keys of one layer brought to unit mean square, per head or across
          all heads of a token, and rotated; K and V go on into the cache (or K stays
          compact).
  kv4     one iteration's part of a layer whose KV cache is kept in 4 bits: the fresh rows
          of the active tokens are quantised into it (K rotated on its way, or not), then
          the whole layer is read back.
  paged4  a few new tokens per sequence against 4-bit caches held in pages: sequences of
          their own lengths, query heads in groups that share a K/V head.

With `own` the calls of this library run; without it the same results come from
elementary torch operations in 32 bits, rounded once.

The 4-bit cache holds a row of D values of one token and head as D e2m1 codes, two to a
byte (the even one low), and a word: six bits each of the factors m_0 .. m_3 from the lowest
bit on, then a byte s.  Dimension d is of group (d / (D/32)) mod 4 and stands for
code * m_group * 2^(s - 127).
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
TOP = 252.0 * 2.0 ** 120    # larger magnitudes count as this in the 4-bit cache


def listed():
    return [
        # 64 sequences with one new token each, a few of them ended: a server's every step.
        {"name": "plan_tokens", "kind": "plan", "batch": 64, "lo": 1, "hi": 4000, "new": 1,
         "ended": 0.1, "page": 16, "keys": False, "mix": 11},
        # 24 prompts continued over their caches, which are read back for the packed
        # attention: the largest plan.
        {"name": "plan_prompts", "kind": "plan", "batch": 24, "lo": 0, "hi": 32000, "new": 3000,
         "ended": 0.1, "page": 64, "keys": True, "mix": 12},
        # One new token of 48 sequences out of a fused projection, K and V into the cache: a
        # decoder's step, all launch latency.
        {"name": "norm_tokens", "kind": "norm", "n": 48, "rows": 65536, "Hq": 32, "Hkv": 8,
         "D": 128, "dtype": "bf16", "across": False, "rope": True, "fused": True},
        # A small fp32 layer (4x16x16 tokens, 4 heads x 64), K kept compact.
        {"name": "norm_tiny_f32", "kind": "norm", "n": 1024, "rows": 0, "Hq": 4, "Hkv": 4, "D": 64,
         "dtype": "f32", "across": False, "rope": True, "fused": False},
        # An LTX-like layer (16x16x24 tokens, 32 heads x 64), three quarters of the tokens
        # active, normed per head: the ordinary iteration.
        {"name": "norm_ltx_most", "kind": "norm", "n": 4608, "rows": 6144, "Hq": 32, "Hkv": 32,
         "D": 64, "dtype": "bf16", "across": False, "rope": True, "fused": True},
        # A Wan-14B-like layer (40 heads x 128) of a 720p-like video (21x45x80 tokens), a
        # quarter of the tokens active, normed across the heads: the largest.
        {"name": "norm_720p_quarter", "kind": "norm", "n": 18900, "rows": 75600, "Hq": 40,
         "Hkv": 40, "D": 128, "dtype": "bf16", "across": True, "rope": True, "fused": False},
        # The small fp32 layer, a quarter of the tokens active: the smallest use.
        {"name": "kv4_tiny_f32", "kind": "kv4", "F": 4, "Hh": 16, "Ww": 16, "H": 4, "D": 64,
         "dtype": "f32", "share": 0.25, "rope": False},
        # The Wan-14B-like layer, a quarter of the tokens active: the largest.
        {"name": "kv4_720p_quarter", "kind": "kv4", "F": 21, "Hh": 45, "Ww": 80, "H": 40,
         "D": 128, "dtype": "bf16", "share": 0.25, "rope": True},
        # One new token of one sequence of 4001: the latency of a single user's step.
        {"name": "token4_one", "kind": "paged4", "batch": 1, "lo": 4001, "hi": 4001, "mix": 1,
         "new": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 16},
        # One new token of 48 sequences of mixed ages: a busy server.
        {"name": "token4_ragged", "kind": "paged4", "batch": 48, "lo": 100, "hi": 9000, "mix": 2,
         "new": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 64},
        # Four sequences of up to 128k tokens: few rows, long caches.
        {"name": "token4_long", "kind": "paged4", "batch": 4, "lo": 60000, "hi": 131072, "mix": 3,
         "new": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 128},
        # Four drafted tokens per sequence, each head with its own K/V (12 heads x 64).
        {"name": "draft4_mha", "kind": "paged4", "batch": 16, "lo": 300, "hi": 12000, "mix": 4,
         "new": 4, "Hq": 12, "Hkv": 12, "D": 64, "page": 32},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "norm", "kv4", "paged4"])
    if kind == "plan":
        batch = _log(rng, 1, 512)
        keys = rng.random() < 0.5
        hi = _log(rng, 2, max(3, min(131072, 150000 // batch)))
        return {"kind": kind, "batch": batch, "lo": int(hi * rng.choice([0.0, 0.1, 0.9])), "hi": hi,
                "new": _log(rng, 1, max(2, min(8000, 30000 // batch))),
                "ended": rng.choice([0.0, 0.1, 0.4]), "page": rng.choice([1, 8, 16, 32, 64, 128, 256]),
                "keys": keys, "mix": rng.randrange(1 << 30)}
    if kind == "norm":
        D = rng.choice([8, 32, 64, 64, 80, 96, 128, 128, 256])
        Hkv = rng.choice([1, 2, 3, 4, 7, 8, 12, 24, 32, 40])
        Hq = min(64, Hkv * rng.choice([1, 1, 2, 4, 8])) // Hkv * Hkv
        n = _log(rng, 1, min(20000, 96_000_000 // (max(Hq, Hkv) * D)))
        return {"kind": kind, "n": n, "rows": rng.choice([0, n, 2 * n + 5]), "Hq": Hq, "Hkv": Hkv,
                "D": D, "dtype": rng.choice(["bf16", "bf16", "f32"]), "across": rng.random() < 0.5,
                "rope": rng.random() < 0.8, "fused": rng.random() < 0.5}
    if kind == "kv4":
        H, D = rng.choice([1, 3, 4, 7, 12, 24, 32, 40]), rng.choice([64, 128])
        n = _log(rng, 300, min(75600, 387_000_000 // (H * D)))
        Hh, Ww = rng.randint(1, 17), rng.randint(1, 17)
        rope = rng.random() < 0.6
        return {"kind": kind, "F": max(1, n // (Hh * Ww)), "Hh": Hh, "Ww": Ww, "H": H, "D": D,
                "dtype": "bf16" if rope or rng.random() < 0.6 else "f32",
                "share": round(rng.uniform(0.05, 0.3), 3), "rope": rope}
    D = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
    hi = _log(rng, 64, 131072)
    batch = _log(rng, 1, max(1.0, min(96.0, 260000.0 * 8 / (hi * Hkv))))
    return {"kind": kind, "batch": batch, "lo": max(1, int(hi * rng.choice([0.02, 0.3, 1.0]))),
            "hi": hi, "mix": rng.randrange(1 << 30), "new": rng.choice([1, 1, 1, 2, 3, 5]),
            "Hq": Hq, "Hkv": Hkv, "D": D, "page": rng.choice([8, 16, 32, 64, 128, 256])}


# ------------------------------------------------------------------ sizes

def _plan_lengths(case):
    """(present, wanted) length of each sequence."""
    r = random.Random(case["mix"])
    out = []
    for _ in range(case["batch"]):
        have = r.randint(case["lo"], case["hi"])
        out.append((have, 0 if r.random() < case["ended"] else have + r.randint(1, case["new"])))
    return out


def _lengths(case):
    r = random.Random(case["mix"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]


def work(case):
    if case["kind"] == "plan":
        P, lens = case["page"], _plan_lengths(case)
        pages = sum(abs(-(-w // P) + -h // P) for h, w in lens)
        new = sum(max(0, w - h) for h, w in lens)
        keys = sum(w for _, w in lens) if case["keys"] else 0
        out = case["batch"] * (8 + 4 + 4 + (4 if case["keys"] else 0))
        # a page moved is read and written once; a token's page is read once per page
        return {"bytes": out + 8 * pages + 8 * new + 4 * keys + 4 * ((new + keys) // P),
                "flops": 4 * new + 4 * keys + 8 * case["batch"]}
    D = case["D"]
    if case["kind"] == "norm":
        n, w = case["n"], 2 if case["dtype"] == "bf16" else 4
        heads = 2 * case["Hq"] + 2 * case["Hkv"] + (2 * case["Hkv"] if case["rows"] else 0)
        return {"bytes": n * heads * D * w + (n * (4 * D + 4) if case["rope"] else 0) +
                (4 * n if case["rows"] else 0),
                "flops": n * (case["Hq"] + case["Hkv"]) * D * (8 if case["rope"] else 4)}
    if case["kind"] == "kv4":
        n_all = case["F"] * case["Hh"] * case["Ww"]
        n = max(1, int(n_all * case["share"]))
        H, w = case["H"], 2 if case["dtype"] == "bf16" else 4
        row = D // 2 + 4
        write = n * (2 * H * D * w + 2 * H * row + 4 + (4 * D if case["rope"] else 0))
        read = n_all * (2 * H * row + 2 * H * D * w)
        return {"bytes": write + read, "flops": (8 if case["rope"] else 4) * n * H * D}
    Hq, Hkv, new, lens = case["Hq"], case["Hkv"], case["new"], _lengths(case)
    pairs = sum(max(0, k - new + i + 1) for k in lens for i in range(new))
    return {"bytes": 2 * sum(lens) * Hkv * (D // 2 + 4) + 2 * case["batch"] * new * Hq * D * 2 +
            4 * sum(-(-k // case["page"]) for k in lens), "flops": 4 * D * Hq * pairs}


# ----------------------------------------------------------------- inputs

def _normal(g, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _keys(g, rows, H, D, dtype=torch.bfloat16):
    """Keys have a few channels that are larger than the others, as trained models' do."""
    k = torch.randn((rows, H, D), generator=g, device=DEV, dtype=torch.float32)
    big = torch.rand((1, H, D), generator=g, device=DEV) < 0.03
    return (k * torch.where(big, 4.0, 0.9)).to(dtype)


def _angles(at, axes_bands):
    """(cos, sin) in 32 bits of positions times frequencies; far positions need 64 bits."""
    a = torch.cat([p[:, None].double() *
                   10000.0 ** (-torch.arange(b, device=DEV).double() / max(b, 1))
                   for p, b in axes_bands], 1)
    return torch.stack([a.cos(), a.sin()], -1).float()


def _power(e):
    """2^e in 32 bits, e an integer tensor in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _groups(D):
    """The group of each dimension."""
    return torch.arange(D, device=DEV) // (D // 32) % 4


def _quantise(x):
    """(codes of two values a byte, words) of the rows x[..., D], in 32 bits; borders by exact
    comparisons."""
    D = x.shape[-1]
    x = x.float().clamp(-TOP, TOP)
    a = x.abs().unflatten(-1, (8, 4, D // 32)).amax((-3, -1))
    f, e = torch.frexp(a.amax(-1))
    e = torch.where(f > 378.0 / 512.0, e - 8, e - 9)      # least e with the largest <= 378 2^e
    e = torch.where(f == 0, torch.full_like(e, -100), e).clamp(min=-100)
    m = torch.ceil((a * _power(-e)[..., None]).double() / 6.0)
    unit = m.float()[..., _groups(D)]
    y = x.abs() * _power(-e)[..., None]
    code = torch.zeros_like(x, dtype=torch.uint8)
    for i, border in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        # between codes i and i + 1; in the middle lies the even one's
        code += (y > unit * border) if i % 2 == 0 else (y >= unit * border) & (unit > 0)
    code |= torch.signbit(x).to(torch.uint8) << 3
    m = m.int()
    word = m[..., 0] | m[..., 1] << 6 | m[..., 2] << 12 | m[..., 3] << 18 | (e.int() + 127) << 24
    return code[..., 0::2] | code[..., 1::2] << 4, word


def _values(pair, word):
    """What codes [..., D/2] with words [...] stand for, in 32 bits."""
    code = torch.stack([pair & 15, pair >> 4], -1).flatten(-2)
    c = (code & 7).int()
    size = torch.where(c < 2, c.float() * 0.5,
                       (2 + (c & 1)).float() * _power((c >> 1) - 2))
    size = torch.where(code > 7, -size, size)
    m = (word[..., None] >> (6 * _groups(code.shape[-1]).int())) & 63
    return size * m.float() * _power((word >> 24 & 255) - 127)[..., None]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 17)
    s = {"case": case}
    if case["kind"] == "plan":
        return _prepare_plan(case, g, s)
    D = case["D"]
    if case["kind"] == "norm":
        return _prepare_norm(case, g, s)
    if case["kind"] == "kv4":
        dt, H = DTYPES[case["dtype"]], case["H"]
        N = case["F"] * case["Hh"] * case["Ww"]
        n = max(1, int(N * case["share"]))
        s["idx"] = torch.randperm(N, generator=g, device=DEV)[:n].sort().values.int()
        s["k_fresh"], s["v_fresh"] = _keys(g, n, H, D, dt), _normal(g, (n, H, D), dt)
        # the layer's cache as the iterations before left it
        for name, x in (("k", _keys(g, N, H, D)), ("v", _normal(g, (N, H, D)))):
            s[name + "_cache"], s[name + "_scale"] = _quantise(x)
            s[name + "_out"] = torch.empty((N, H, D), dtype=dt, device=DEV)
        s["table"] = None
        if case["rope"]:
            at = torch.arange(N, device=DEV)
            s["table"] = _angles(at, ((at // (case["Hh"] * case["Ww"]), D // 2 - 2 * (D // 6)),
                                      (at // case["Ww"] % case["Hh"], D // 6),
                                      (at % case["Ww"], D // 6)))
        return s
    P, B, lens = case["page"], case["batch"], _lengths(case)
    s["lens"] = lens
    need = [-(-k // P) for k in lens]
    pages = sum(need) + 3
    ids = torch.randperm(pages, generator=g, device=DEV).int()
    s["table"] = torch.zeros((B, max(need)), dtype=torch.int32, device=DEV)
    at = 0
    for b, c in enumerate(need):
        s["table"][b, :c] = ids[at:at + c]
        at += c
    s["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["q"] = _normal(g, (B, case["new"], case["Hq"], D))
    for name, make in (("k", _keys), ("v", lambda g, r, h, d: _normal(g, (r, h, d)))):
        x = make(g, pages * P, case["Hkv"], D).view(pages, P, case["Hkv"], D)
        s[name + "_pages"], s[name + "_scale"] = _quantise(x)
    s["out"] = torch.empty_like(s["q"])
    s["workspace"] = None
    return s


def _prepare_plan(case, g, s):
    P, B, lens = case["page"], case["batch"], _plan_lengths(case)
    have, need = ([-(-x[i] // P) for x in lens] for i in (0, 1))
    most = max(max(have), max(need))
    spare = sum(max(0, b - a) for a, b in zip(have, need)) + 5
    pages = sum(have) + spare
    ids = torch.randperm(pages, generator=g, device=DEV).int()
    # which pages a sequence holds says the order of the identifiers
    j = torch.arange(most, device=DEV)
    held = torch.tensor(have, device=DEV)
    first = held.cumsum(0) - held
    at = (first[:, None] + j).clamp(max=pages - 1)
    s["table"] = torch.where(j < held[:, None], ids[at], torch.zeros_like(ids[at])).contiguous()
    s["free"] = torch.cat([ids[sum(have):], torch.full((sum(have),), -7, dtype=torch.int32,
                                                       device=DEV)])
    s["n_free"] = torch.tensor([spare], dtype=torch.int32, device=DEV)
    s["n_free_out"] = torch.zeros_like(s["n_free"])
    s["lens"], s["want"] = (torch.tensor([x[i] for x in lens], dtype=torch.int32, device=DEV)
                            for i in (0, 1))
    s["lens_out"] = torch.zeros_like(s["lens"])
    s["cu_q"], s["cu_k"] = (torch.zeros(B + 1, dtype=torch.int32, device=DEV) for _ in "qk")
    new = sum(max(0, b - a) for a, b in lens)
    # a batch has room to spare, as one of a fixed size that a graph holds
    s["slots"], s["positions"] = (torch.zeros(new + new // 8 + 3, dtype=torch.int32, device=DEV)
                                  for _ in "sp")
    s["rows"] = torch.zeros(sum(b for _, b in lens) + 7, dtype=torch.int32, device=DEV)
    return s


def _prepare_norm(case, g, s):
    n, Hq, Hkv, D, N = case["n"], case["Hq"], case["Hkv"], case["D"], case["rows"]
    dt = DTYPES[case["dtype"]]
    parts = (_normal(g, (n, Hq, D)) * 1.7, _keys(g, n, Hkv, D), _normal(g, (n, Hkv, D)))
    if case["fused"]:
        all_of = torch.cat(parts, 1).to(dt)
        s["q"], s["k"], s["v"] = all_of.split((Hq, Hkv, Hkv), 1)
    else:
        s["q"], s["k"], s["v"] = (x.to(dt) for x in parts)
    for name, H in (("q", Hq), ("k", Hkv)):
        shape = (H, D) if case["across"] else (D,)
        s[name + "_weight"] = 1 + 0.2 * torch.randn(shape, generator=g, device=DEV)
    s["q_out"] = torch.empty((n, Hq, D), dtype=dt, device=DEV)
    s["idx"] = None
    if N:
        s["idx"] = torch.randperm(N, generator=g, device=DEV)[:n].int()
        s["k_out"], s["v_out"] = (_normal(g, (N, Hkv, D), dt) for _ in "kv")
    else:
        s["k_out"], s["v"], s["v_out"] = torch.empty((n, Hkv, D), dtype=dt, device=DEV), None, None
    s["table"] = s["at"] = None
    if case["rope"]:
        far = 8192
        s["table"] = _angles(None, ((torch.arange(far, device=DEV), D // 2),))
        s["at"] = torch.randint(0, far, (n,), generator=g, device=DEV).int()
    return s


# -------------------------------------------------------------------- run

def run(s):
    if own:
        return _run_own(s)
    return {"plan": _plan, "norm": _norm, "kv4": _kv4, "paged4": _paged}[s["case"]["kind"]](s)


def _plan_outputs(s):
    out = {name: s[name] for name in ("table", "free", "n_free_out", "lens_out", "cu_q", "slots",
                                      "positions")}
    return {**out, "cu_k": s["cu_k"], "rows": s["rows"]} if s["case"]["keys"] else out


def _norm_outputs(s):
    out = {"q": s["q_out"], "k": s["k_out"]}
    return {**out, "v": s["v_out"]} if s["v"] is not None else out


def _run_own(s):
    import paper_2605_06892_gb300 as hsa
    c = s["case"]
    if c["kind"] == "plan":
        more = {"cu_k": s["cu_k"], "key_rows": s["rows"]} if c["keys"] else {}
        hsa.hsa_page_plan(s["lens"], s["want"], c["page"], s["table"], s["free"], s["n_free"],
                          s["n_free_out"], s["lens_out"], s["cu_q"], s["slots"], s["positions"],
                          **more)
        return _plan_outputs(s)
    if c["kind"] == "norm":
        hsa.hsa_qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["q_out"], s["k_out"],
                             eps=EPS, across=c["across"], table=s["table"], table_idx=s["at"],
                             v=s["v"], v_out=s["v_out"], k_idx=s["idx"])
        return _norm_outputs(s)
    if c["kind"] == "kv4":
        n, N = s["idx"].numel(), s["k_cache"].shape[0]
        hsa.hsa_kv4_quant_scatter(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                                  s["k_fresh"], s["v_fresh"], s["idx"], n, table=s["table"])
        hsa.hsa_kv4_dequant_gather(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], None,
                                   N, s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"], "k_scale": s["k_scale"],
                "v_scale": s["v_scale"]}
    if s["workspace"] is None:   # once, kept as a user's program keeps it
        size = hsa.hsa_paged_attention_workspace_bytes(c["batch"], c["new"], c["Hq"], c["Hkv"],
                                                       c["D"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    hsa.hsa_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["seq_lens"],
                            s["out"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                            workspace=s["workspace"])
    return s["out"]


def _plan(s):
    P, table, free = s["case"]["page"], s["table"], s["free"]
    B, cols = table.shape
    have_tok, want = s["lens"].long(), s["want"].long()
    have, need = (have_tok + P - 1) // P, (want + P - 1) // P
    back, get = (have - need).clamp(min=0), (need - have).clamp(min=0)
    new = (want - have_tok).clamp(min=0)
    count = s["n_free"].long() + back.sum()
    # sequences grow in their order while pages and places for tokens last
    ok = ((get.cumsum(0) <= count) | (get == 0)) & (new.cumsum(0) <= s["slots"].numel()) | (new == 0)
    get, new = get * ok, new * ok
    s["lens_out"].copy_(torch.where(ok, want, have_tok))
    s["n_free_out"].copy_(count - get.sum())
    j = torch.arange(cols, device=DEV)
    flat = table.flatten()
    # pages given back go onto the stack, in order; the element behind it takes the rest
    rank = (back.cumsum(0) - back)[:, None] + j - need[:, None]
    leaves = (j >= need[:, None]) & (j < have[:, None])
    ext = torch.cat([free, free[:1]])
    ext[torch.where(leaves, s["n_free"] + rank, free.numel()).flatten()] = flat
    free.copy_(ext[:-1])
    # pages taken come from its top
    rank = (get.cumsum(0) - get)[:, None] + j - have[:, None]
    comes = (j >= have[:, None]) & (j < (have + get)[:, None])
    taken = free[torch.where(comes, count - 1 - rank, 0)]
    table.copy_(torch.where(comes, taken, table))
    s["cu_q"][1:] = new.cumsum(0)

    def rows(ends, total, first):
        i = torch.arange(total, device=DEV)
        b = torch.searchsorted(ends[1:].contiguous(), i, right=True)
        there = b < B
        b = b.clamp(max=B - 1)
        at = torch.where(there, i - ends[b] + first[b], 0)
        return (torch.where(there, table[b, at // P].long() * P + at % P, -1),
                torch.where(there, at, -1))
    slots, positions = rows(s["cu_q"].long(), s["slots"].numel(), have_tok)
    s["slots"].copy_(slots)
    s["positions"].copy_(positions)
    if s["case"]["keys"]:
        s["cu_k"][1:] = s["lens_out"].long().cumsum(0)
        s["rows"].copy_(rows(s["cu_k"].long(), s["rows"].numel(), torch.zeros_like(want))[0])
    return _plan_outputs(s)


def _norm(s):
    c = s["case"]
    out = []
    for name in ("q", "k"):
        x = s[name].float()
        over = (-2, -1) if c["across"] else (-1,)
        x = x * torch.rsqrt((x * x).mean(over, keepdim=True) + EPS) * s[name + "_weight"]
        if c["rope"]:
            cs, sn = (y[:, None] for y in s["table"][s["at"].long()].unbind(-1))
            x0, x1 = x[..., 0::2], x[..., 1::2]
            x = torch.stack([x0 * cs - x1 * sn, x0 * sn + x1 * cs], -1).flatten(-2)
        out.append(x.to(s["q_out"].dtype))
    s["q_out"].copy_(out[0])
    if s["idx"] is None:
        s["k_out"].copy_(out[1])
    else:
        s["k_out"][s["idx"].long()] = out[1]
        s["v_out"][s["idx"].long()] = s["v"]
    return _norm_outputs(s)


def _kv4(s):
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
        s[name + "_cache"][idx], s[name + "_scale"][idx] = _quantise(x)
        out[name] = _values(s[name + "_cache"], s[name + "_scale"]).to(s[name + "_out"].dtype)
        out[name + "_scale"] = s[name + "_scale"]
    return out


def _paged(s):
    c = s["case"]
    q = s["q"].unflatten(2, (c["Hkv"], -1)).float()
    out = torch.empty_like(s["q"])
    for b, n in enumerate(s["lens"]):
        ids = s["table"][b, :-(-n // c["page"])].long()
        k, v = (_values(s[x + "_pages"][ids], s[x + "_scale"][ids]).flatten(0, 1)[:n].transpose(0, 1)
                for x in ("k", "v"))
        rows = q[b].permute(1, 0, 2, 3).flatten(1, 2)           # [Hkv, new G, D]
        x = torch.matmul(rows, k.transpose(1, 2)) / math.sqrt(c["D"])
        i = torch.arange(c["new"], device=DEV).repeat_interleave(q.shape[3])
        seen = torch.arange(n, device=DEV) < (n - c["new"] + 1 + i)[:, None]
        x = x.masked_fill_(~seen, -math.inf)
        x = torch.exp(x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)))
        total = x.sum(-1, keepdim=True)
        o = torch.matmul(x, v) / torch.where(total > 0, total, torch.ones_like(total))
        out[b] = o.unflatten(1, (c["new"], -1)).permute(1, 0, 2, 3).flatten(1, 2)
    return out


# ------------------------------------------------------------------ exact

def _rounded(x, bits, least):
    """64-bit values to `bits` significant bits, ties to even; steps of 2^least at least."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - bits).clamp(min=least).double())
    return torch.round(x / step) * step


def _exact_rows(x):
    """Values and words that the 4-bit cache holds for the 64-bit rows x."""
    D = x.shape[-1]
    x = x.clamp(-TOP, TOP)
    # a group's dimensions: every fourth run of D / 32
    of = [torch.cat([torch.arange(r, r + D // 32) for r in range(h * (D // 32), D, D // 8)])
          for h in range(4)]
    a = torch.stack([x[..., i].abs().amax(-1) for i in of], -1)
    most = a.amax(-1)
    e = torch.ceil(torch.log2(most.clamp(min=1e-300) / 378.0))
    e = torch.where(most * torch.exp2(-e) > 378.0, e + 1, e)     # the logarithm's own rounding
    e = torch.where(most * torch.exp2(1 - e) <= 378.0, e - 1, e).clamp(min=-100.0)
    m = torch.ceil(a / (6.0 * torch.exp2(e))[..., None])
    out = torch.zeros_like(x)
    word = (e + 127).long() << 24
    for h, i in enumerate(of):
        unit = (m[..., h] * torch.exp2(e))[..., None]
        out[..., i] = torch.where(unit > 0, _rounded(x[..., i] / unit, 2, -1) * unit, 0.0)
        word |= m[..., h].long() << (6 * h)
    return out, torch.where(word >= 1 << 31, word - (1 << 32), word).int()


_CODES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_values(pair, word):
    D = 2 * pair.shape[-1]
    code = torch.empty((*pair.shape[:-1], D), dtype=torch.int32, device=DEV)
    code[..., 0::2], code[..., 1::2] = pair.int() % 16, pair.int() // 16
    x = torch.tensor(_CODES + [-c for c in _CODES], dtype=torch.float64, device=DEV)[code]
    bits = word.long() & 0xffffffff
    for d in range(0, D, D // 32):
        h = d // (D // 32) % 4
        x[..., d:d + D // 32] *= (torch.exp2((bits >> 24).double() - 127) *
                                  (bits >> (6 * h) & 63))[..., None]
    return x


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "norm": _exact_norm, "kv4": _exact_kv4,
            "paged4": _exact_paged}[case["kind"]](s)


def _exact_plan(s):
    """One sequence after another, on the host."""
    P = s["case"]["page"]
    table, free = s["table"].cpu().clone(), s["free"].cpu().clone()
    lens, want, top = s["lens"].tolist(), s["want"].tolist(), int(s["n_free"])
    after = list(lens)
    for b, (h, w) in enumerate(zip(lens, want)):
        if w < h:
            for j in range(-(-w // P), -(-h // P)):
                free[top] = table[b, j]
                top += 1
            after[b] = w
    cu_q, tok, rows = [0], [], []
    for b, (h, w) in enumerate(zip(lens, want)):
        if w > h:
            for j in range(-(-h // P), -(-w // P)):
                top -= 1
                table[b, j] = free[top]
            p = torch.arange(h, w)
            tok.append((table[b, p // P].long() * P + p % P, p))
            after[b] = w
        cu_q.append(cu_q[-1] + max(0, w - h))
        p = torch.arange(after[b])
        rows.append(table[b, p // P].long() * P + p % P)

    def filled(parts, size):
        x = torch.cat(parts + [torch.full((size,), -1)])[:size]
        return x.int().to(DEV)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)
    out = {"table": table.to(DEV), "free": free.to(DEV), "n_free_out": ints([top]),
           "lens_out": ints(after), "cu_q": ints(cu_q),
           "slots": filled([t[0] for t in tok], s["slots"].numel()),
           "positions": filled([t[1] for t in tok], s["positions"].numel())}
    if s["case"]["keys"]:
        cu_k = [0]
        for n in after:
            cu_k.append(cu_k[-1] + n)
        out["cu_k"], out["rows"] = ints(cu_k), filled(rows, s["rows"].numel())
    return out


def _exact_norm(s):
    c, out = s["case"], {}
    for name in ("q", "k"):
        x = s[name].double()
        n, H, D = x.shape
        rows = x.reshape(n, 1, H * D) if c["across"] else x
        unit = (rows.square().sum(-1, keepdim=True) / rows.shape[-1] + EPS).sqrt()
        x = (rows / unit).view(n, H, D) * s[name + "_weight"].double()
        if c["rope"]:
            turn = torch.view_as_complex(s["table"].double())[s["at"].long()][:, None]
            x = torch.view_as_real(torch.view_as_complex(x.view(n, H, D // 2, 2)) * turn).view(n, H, D)
        out[name] = x
    if s["idx"] is not None:
        for name, x in (("k", out["k"]), ("v", s["v"].double())):
            out[name] = s[name + "_out"].double()
            out[name][s["idx"].long()] = x
    return out


def _exact_kv4(s):
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
        held, word = _exact_values(s[name + "_cache"], s[name + "_scale"]), s[name + "_scale"].clone()
        held[idx], word[idx] = _exact_rows(x)
        out[name], out[name + "_scale"] = held, word
    return out


def _exact_paged(s):
    c = s["case"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    G = c["Hq"] // c["Hkv"]
    for b, n in enumerate(s["lens"]):
        at = torch.arange(n, device=DEV)
        page, row = s["table"][b, at // c["page"]].long(), at % c["page"]
        k, v = (_exact_values(s[x + "_pages"][page, row], s[x + "_scale"][page, row])
                for x in ("k", "v"))
        for i in range(c["new"]):
            m = n - c["new"] + i + 1
            if m <= 0:
                continue
            for h in range(c["Hq"]):
                x = k[:m, h // G] @ s["q"][b, i, h].double() * c["D"] ** -0.5
                out[b, i, h] = torch.softmax(x, 0) @ v[:m, h // G]
    return out
