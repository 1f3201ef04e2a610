"""Plain 64-bit references of the 8-bit KV cache and of attention over packed or paged
sequences with grouped heads, on the CPU, from the definitions in include/hsa.h; and the
error that a kernel's roundings may make, term by term."""
import numpy as np
import torch

LEAST = -100                     # smallest exponent of a row's power of two
TOP = 1.875 * 2.0 ** 127         # larger finite magnitudes count as this


def e4m3_table():
    """Value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 fraction bits;
    0x7f and 0xff are NaN."""
    v = np.zeros(256)
    for c in range(256):
        s, e, f = c >> 7, (c >> 3) & 15, c & 7
        x = f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        v[c] = np.nan if c & 0x7f == 0x7f else (-x if s else x)
    return v


VALUES = e4m3_table()


def quantise_rows(x):
    """(codes, scale bytes, any non-finite) of float64 rows x[..., D]."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    y = np.where(finite, np.clip(x, -TOP, TOP), 0.0)
    a = np.abs(y).max(-1)
    e = np.full(a.shape, LEAST, dtype=np.int64)
    for i in np.ndindex(a.shape):
        while a[i] * 2.0 ** -float(e[i]) > 448.0:
            e[i] += 1
    y = y * np.exp2(-e.astype(np.float64))[..., None]
    # nearest of the 127 magnitudes, ties to the even fraction
    grid = VALUES[:127]
    at = np.clip(np.searchsorted(grid, np.abs(y)), 1, 126)
    lo, hi = grid[at - 1], grid[at]
    up = (np.abs(y) - lo > hi - np.abs(y)) | ((np.abs(y) - lo == hi - np.abs(y)) & (at % 2 == 0))
    code = np.where(up, at, at - 1).astype(np.int64)
    code = np.where(np.signbit(x) & finite, code | 0x80, code)
    return np.where(finite, code, 0x7f), (e + 127).astype(np.uint8), not finite.all()


def values(code, scale):
    """What codes [..., D] (uint8) with scale bytes [...] stand for, float64."""
    return VALUES[np.asarray(code).astype(np.int64)] * np.exp2(
        np.asarray(scale).astype(np.float64) - 127)[..., None]


def limits(lq, lk, mask):
    """Keys that each of the lq newest of lk tokens may see; mask as in hsa_packed_attention."""
    p = np.arange(lq) + lk - lq
    return np.full(lq, lk) if not mask else np.clip((p // mask + 1) * mask, 0, lk)


def attention(q, k, v, limit, scale=None, p_step=2.0 ** -8, out_step=2.0 ** -8):
    """q [n, Hq, D] against k, v [m, Hkv, D] (float64 tensors), row i over its first limit[i]
    keys only.  Returns (out, tolerance): out is rounded by at most out_step of itself; each
    probability by p_step; a score, a sum of D products in 32 bits, is off by at most
    (D + 2) 2^-24 of the sum of its products' magnitudes, which moves its probability by
    that much, and the normalising sum by as much again; 2^-21 covers the exponential
    (2^-22.5) and the 32-bit sums over the keys, which the kernels split into short runs."""
    n, Hq, D = q.shape
    m, Hkv = k.shape[0], k.shape[1] if k.dim() == 3 else 1
    scale = D ** -0.5 if scale is None else scale
    out, tol = torch.zeros((n, Hq, D), dtype=torch.float64), torch.zeros((n, Hq, D), dtype=torch.float64)
    for h in range(Hq):
        kh, vh = k[:, h * Hkv // Hq], v[:, h * Hkv // Hq]
        for i in range(n):
            c = int(limit[i])
            if c <= 0:
                continue
            s = (kh[:c] @ q[i, h]) * scale
            w = torch.softmax(s, 0)
            out[i, h] = w @ vh[:c]
            slack = float((kh[:c].abs() @ q[i, h].abs()).max()) * scale * (D + 2) * 2.0 ** -24
            spread = w @ vh[:c].abs()
            tol[i, h] = out_step * out[i, h].abs() + (p_step + 2 * slack + 2.0 ** -21) * spread
    return out, tol + 1e-30
