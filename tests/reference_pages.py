"""Plain references of the 4-bit KV cache (64 bits), of the normed and rotated rows (64 bits)
and of the page plan (one sequence after another), on the CPU, from the definitions in
include/hsa.h."""
import numpy as np
import torch

LEAST = -100                       # smallest exponent of a row
TOP = 252.0 * 2.0 ** 120           # larger finite magnitudes count as this
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NAN_ROW = 0xff000000


def group_of(D):
    return np.arange(D) // (D // 32) % 4


def encode_rows(x):
    """(codes of two a byte, words, any row not finite) of float64 rows x[..., D].  Products of
    numbers of few bits are exact, so every border is decided by exact comparisons."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x).all(-1)
    g = group_of(x.shape[-1])
    y = np.where(finite[..., None], np.clip(x, -TOP, TOP), 0.0)
    a = np.stack([np.abs(y[..., g == h]).max(-1) for h in range(4)], -1)
    top = a.max(-1)
    e = np.full(top.shape, LEAST, dtype=np.int64)
    while (more := top > 378.0 * np.exp2(e.astype(float))).any():
        e += more
    m = np.zeros(a.shape, dtype=np.int64)
    while (more := a > 6.0 * m * np.exp2(e.astype(float))[..., None]).any():
        m += more
    unit = (m * np.exp2(e.astype(float))[..., None])[..., g]
    code = np.zeros(x.shape, dtype=np.int64)
    for i in range(7):
        border = (GRID[i] + GRID[i + 1]) / 2 * unit
        # a tie goes to the even code
        code += (np.abs(y) > border) | ((np.abs(y) == border) & (i % 2 == 1) & (unit > 0))
    code += 8 * np.signbit(y)
    word = (e + 127) << 24
    for h in range(4):
        word |= m[..., h] << (6 * h)
    pair = (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)
    return (np.where(finite[..., None], pair, 0).astype(np.uint8),
            np.where(finite, word, NAN_ROW).astype(np.uint32), not finite.all())


def quantise_rows(x):
    """(values held, words, any row not finite) of float64 rows x[..., D]."""
    pair, word, odd = encode_rows(x)
    return values(pair, word), word, odd


def values(pair, word):
    """What codes [..., D/2] (uint8) with words [...] (int32 or uint32) stand for, float64."""
    pair = np.asarray(pair).astype(np.int64)
    word = np.asarray(word).astype(np.int64) & 0xffffffff
    code = np.stack([pair & 15, pair >> 4], -1).reshape(*pair.shape[:-1], 2 * pair.shape[-1])
    m = word[..., None] >> (6 * group_of(code.shape[-1])) & 63
    s = (word >> 24)[..., None]
    v = np.where(code > 7, -GRID[code & 7], GRID[code & 7]) * m * np.exp2(s - 127.0)
    return np.where(s == 255, np.nan, v)


def norm_rope(x, weight, eps, across, table, rows, out_step):
    """(out, tolerance) of rows x [n, H, D]; table [.., D/2, 2] by `rows`, or None.  The result
    is rounded by out_step of itself.  In 32 bits: the square sum's additions (at most 8 in a
    lane and 8 across lanes; 32, 8 and 32 for a whole row), half of them in the root; the mean
    and eps three more, so halved; the root itself, two products, and two of the rotation, each
    2^-24 of the terms' magnitudes."""
    x = x.double()
    n, H, D = x.shape
    flat = x.reshape(n, 1, H * D) if across else x
    steps = (72 if across else 16) / 2 + 2 + 3 + 2
    y = (flat / (flat.square().mean(-1, keepdim=True) + eps).sqrt()).reshape(n, H, D)
    if weight is not None:
        y = y * weight.double()
    size = y.abs()
    if table is not None:
        c, s = (table[rows.long()][:, None, :, i].double() for i in (0, 1))
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
        a, b = a.abs(), b.abs()
        size = torch.stack([a * c.abs() + b * s.abs(), a * s.abs() + b * c.abs()], -1).flatten(-2)
    return y, out_step * y.abs() + steps * 2.0 ** -24 * size + 1e-38


# A 4-bit attention's probabilities are rounded to fp16 and again after a factor of a group: at
# most 2^-11 of themselves each.
P_STEP = 2.0 ** -10 + 2.0 ** -22


def small_weights(q, k, v_word, limit, scale=None):
    """What the fp16 probabilities may lose below their normal range [n, Hq, 1]: a key's weight
    times the power of two of its value row is held within 2^-31 of the largest such product, and
    its product with a factor again; each meets a factor of up to 63 and a code of up to 6."""
    n, Hq, D = q.shape
    m, Hkv = k.shape[:2]
    scale = D ** -0.5 if scale is None else scale
    power = torch.from_numpy(np.exp2((np.asarray(v_word).astype(np.int64) >> 24 & 255) - 127.0))
    out = torch.zeros((n, Hq, 1), dtype=torch.float64)
    for h in range(Hq):
        for i in range(n):
            c = int(limit[i])
            if c > 0:
                w = torch.softmax((k[:c, h * Hkv // Hq] @ q[i, h]) * scale, 0)
                out[i, h] = c * 2.0 ** -31 * (378 + 6) * (w * power[:c, h * Hkv // Hq]).max()
    return out


MOST = 2 ** 31 - 1


def plan(lens, want, page, table, free, n_free, max_new, max_keys=None):
    """The state after the step, as a dict of int32 tensors, and whether an error is
    reported.  table [B, cols], free [pages]."""
    table, free = table.clone(), free.clone()
    B, cols = table.shape
    pages, most = free.numel(), cols * page
    bad = any(not 0 <= x <= most for x in lens + want) or not 0 <= n_free <= pages
    lens, want = ([min(max(x, 0), most) for x in y] for y in (lens, want))
    top = min(max(n_free, 0), pages)

    def up(n):
        return -(-n // page)
    for b in range(B):
        for j in range(up(want[b]), up(lens[b])):
            id_ = int(table[b, j])
            bad |= not 0 <= id_ < pages or top >= pages
            if top < pages:
                free[top] = id_
                top += 1
    after, cu_q, cu_k, tokens, asked, got = [], [0], [0], [], 0, 0
    count = top
    for b in range(B):
        ok = True
        if want[b] > lens[b]:
            get = max(0, up(want[b]) - up(lens[b]))
            asked, got = asked + want[b] - lens[b], got + get
            ok = (get == 0 or got <= count) and asked <= max_new
            if ok:
                for j in range(up(lens[b]), up(want[b])):
                    top -= 1
                    table[b, j] = free[top]
                    bad |= not 0 <= int(free[top]) < pages
        after.append(want[b] if ok else lens[b])
        new = range(lens[b], after[b])
        tokens += [(b, p) for p in new]
        cu_q.append(cu_q[-1] + len(new))
        cu_k.append(min(cu_k[-1] + after[b], MOST))

    def row(b, p):
        nonlocal bad
        id_ = int(table[b, p // page])
        if not 0 <= id_ < pages:
            bad = True
            return -1
        return id_ * page + p % page
    tail = [-1] * (max_new - len(tokens))
    out = {"table": table, "free": free, "n_free_out": [top], "lens_out": after, "cu_q": cu_q,
           "cu_k": cu_k, "slots": [row(b, p) for b, p in tokens] + tail,
           "positions": [p for _, p in tokens] + tail}
    if max_keys is not None:
        rows = []
        for b in range(B):
            for p in range(after[b]):
                if len(rows) == max_keys:
                    bad = True
                    break
                rows.append(row(b, p))
        out["key_rows"] = rows + [-1] * (max_keys - len(rows))
    return {k: torch.as_tensor(v, dtype=torch.int32) for k, v in out.items()}, bad
