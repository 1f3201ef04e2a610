"""Queries and keys normed and rotated, K and V on into the cache (hsa_qk_norm_rope), against
the 64-bit reference."""
import pytest
import torch

import oracle
import reference_pages as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def hsa():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2605_06892_gb300 as m
    m.lib()
    torch.cuda.set_device(0)
    m.hsa_get_device_error()
    return m


def _inputs(n, Hq, Hkv, D, dtype, seed, across):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn((n, H, D), generator=g) for H in (Hq, Hkv, Hkv))
    q = q * torch.exp2(torch.randint(-12, 12, (n, 1, 1), generator=g).float())
    k = k * torch.where(torch.rand((1, Hkv, D), generator=g) < 0.05, 30.0, 1.0)
    q[::7] = 0.0
    w = [1 + 0.3 * torch.randn((H, D) if across else (D,), generator=g) for H in (Hq, Hkv)]
    angle = torch.randn((n + 9, D // 2), generator=g) * 10
    return ([x.to(dtype) for x in (q, k, v)], w, torch.stack([angle.cos(), angle.sin()], -1),
            torch.randperm(n + 9, generator=g)[:n].int(), torch.randperm(2 * n + 3, generator=g)[:n].int())


def _close(got, want, tol):
    err = (got.cpu().double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


SHAPES = [(1, 1, 1, 8), (5, 3, 1, 64), (33, 8, 2, 128), (7, 12, 12, 96), (64, 5, 5, 256), (200, 32, 8, 64),
          (3, 7, 7, 40), (9, 32, 8, 16), (17, 40, 40, 128)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("across", [False, True])
@pytest.mark.parametrize("n,Hq,Hkv,D", SHAPES)
def test_into_the_cache(hsa, n, Hq, Hkv, D, across, dtype):
    """Out of a fused projection, by positions, K and V to rows of a cache; rows of the cache
    that no index names stay."""
    (q, k, v), w, table, at, idx = _inputs(n, Hq, Hkv, D, dtype, 7 * n + D, across)
    wide = torch.cat([q, k, v], 1).to(DEV)
    kc, vc = (torch.full((2 * n + 3, Hkv, D), 3.0, dtype=dtype, device=DEV) for _ in "kv")
    qo = torch.empty((n, Hq, D), dtype=dtype, device=DEV)
    parts = wide.split((Hq, Hkv, Hkv), 1)
    hsa.hsa_qk_norm_rope(parts[0], parts[1], w[0].to(DEV), w[1].to(DEV), qo, kc, eps=1e-6, across=across,
                         table=table.to(DEV), table_idx=at.to(DEV), v=parts[2], v_out=vc, k_idx=idx.to(DEV))
    for got, x, weight in ((qo, q, w[0]), (kc[idx.long()], k, w[1])):
        _close(got, *ref.norm_rope(x, weight, 1e-6, across, table, at, STEP[dtype]))
    assert torch.equal(vc[idx.long()].cpu(), v)
    rest = torch.ones(2 * n + 3, dtype=torch.bool)
    rest[idx.long()] = False
    assert (kc[rest] == 3).all() and (vc[rest] == 3).all()
    assert hsa.hsa_get_device_error() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("across", [False, True])
def test_in_place_and_without_parts(hsa, across, dtype):
    """Compact rows in place; no weights, no table, no V; a table by row or by the cache's row."""
    n, Hq, Hkv, D = 45, 6, 2, 64
    (q, k, v), w, table, at, idx = _inputs(n, Hq, Hkv, D, dtype, 3, across)
    dq, dk = q.to(DEV), k.to(DEV)
    hsa.hsa_qk_norm_rope(dq, dk, None, None, dq, dk, eps=0.5, across=across)
    _close(dq, *ref.norm_rope(q, None, 0.5, across, None, None, STEP[dtype]))
    _close(dk, *ref.norm_rope(k, None, 0.5, across, None, None, STEP[dtype]))
    dq, dk, dv = q.to(DEV), k.to(DEV), v.to(DEV)
    vo = torch.empty_like(dv)
    hsa.hsa_qk_norm_rope(dq, dk, None, w[1].to(DEV), dq, dk, across=across, table=table.to(DEV), v=dv, v_out=vo)
    rows = torch.arange(n)
    _close(dq, *ref.norm_rope(q, None, 1e-6, across, table, rows, STEP[dtype]))
    _close(dk, *ref.norm_rope(k, w[1], 1e-6, across, table, rows, STEP[dtype]))
    assert torch.equal(vo, dv)
    wide = torch.randn((2 * n + 3, D // 2, 2), generator=torch.Generator().manual_seed(1))
    kc = torch.zeros((1, 2 * n + 3, Hkv, D), dtype=dtype, device=DEV)   # one page
    hsa.hsa_qk_norm_rope(q.to(DEV), k.to(DEV), None, None, dq, kc, across=across, table=wide.to(DEV),
                         k_idx=idx.to(DEV))
    _close(dq, *ref.norm_rope(q, None, 1e-6, across, wide, idx, STEP[dtype]))
    _close(kc[0][idx.long()], *ref.norm_rope(k, None, 1e-6, across, wide, idx, STEP[dtype]))
    assert hsa.hsa_get_device_error() == 0


@pytest.mark.parametrize("across", [False, True])
def test_places_without_tokens_and_bad_ones(hsa, across):
    n, H, D, N = 40, 2, 64, 50
    (q, k, v), w, table, at, _ = _inputs(n, H, H, D, torch.bfloat16, 5, across)
    idx = torch.arange(N - 1, N - 1 - n, -1, dtype=torch.int32)
    idx[3], at[8] = -1, -1
    for bad in (False, True):
        if bad:
            idx[11], idx[12], at[20], at[21] = N, -2, table.shape[0], -9
        qo = torch.full((n, H, D), 5.0, dtype=torch.bfloat16, device=DEV)
        kc, vc = (torch.full((N, H, D), 3.0, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        hsa.hsa_qk_norm_rope(q.to(DEV), k.to(DEV), None, None, qo, kc, across=across, table=table.to(DEV),
                             table_idx=at.to(DEV), v=v.to(DEV), v_out=vc, k_idx=idx.to(DEV))
        assert hsa.hsa_get_device_error() == (-6 if bad else 0)
        turned = (at >= 0) & (at < table.shape[0])
        there = turned & (idx >= 0) & (idx < N)
        safe = at.clamp(min=0, max=table.shape[0] - 1)
        want, tol = ref.norm_rope(q, None, 1e-6, across, table, safe, 2.0 ** -8)
        _close(qo, torch.where(turned[:, None, None], want, 5.0), tol)
        want, tol = ref.norm_rope(k, None, 1e-6, across, table, safe, 2.0 ** -8)
        full = torch.full((N, H, D), 3.0, dtype=torch.float64)
        full_tol = torch.zeros_like(full)
        full[idx[there].long()], full_tol[idx[there].long()] = want[there], tol[there]
        _close(kc, full, full_tol)
        full[idx[there].long()] = v[there].double()
        assert torch.equal(vc.cpu().double(), full)


@pytest.mark.parametrize("across", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sizes_of_values(hsa, across, dtype):
    """Values whose squares overflow or vanish in 32 bits, beside ordinary rows."""
    n, H, D = 12, 3, 64
    g = torch.Generator().manual_seed(8)
    x = torch.randn((n, H, D), generator=g).double()
    size = torch.tensor([1e19, 3e19, 1e20, 1e30, 1e38, 1e-20, 1e-25, 1e-38, 1.0, 1e10, 5e18, 2e37])
    x = (x / x.abs().amax((1, 2), keepdim=True) * size.double()[:, None, None]).to(dtype)
    w = torch.ones((H, D) if across else (D,))
    for eps in (1e-6, 1e-30):
        qo, ko = (torch.empty((n, H, D), dtype=dtype, device=DEV) for _ in "qk")
        hsa.hsa_qk_norm_rope(x.to(DEV), x.to(DEV), w.to(DEV), None, qo, ko, eps=eps, across=across)
        eps32 = float(torch.tensor(eps, dtype=torch.float32))
        want, tol = ref.norm_rope(x, None, eps32, across, None, None, STEP[dtype])
        # squares below 2^-126 keep an absolute 2^-149 each: of eps 2^-99 that is 2^-50
        _close(qo, want, tol + 1e-37)
        assert torch.equal(qo, ko)


@pytest.mark.parametrize("across", [False, True])
def test_values_that_are_not_finite(hsa, across):
    """As the formula has it: an infinity makes itself NaN and the other values of its mean zero,
    a NaN the whole mean."""
    n, H, D = 6, 2, 64
    x = torch.randn((n, H, D), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    x[1, 0, 5], x[2, 1, 7], x[4, 0, 0] = float("inf"), float("nan"), float("-inf")
    qo, ko = (torch.empty((n, H, D), dtype=torch.bfloat16, device=DEV) for _ in "qk")
    hsa.hsa_qk_norm_rope(x.to(DEV), x.to(DEV), None, None, qo, ko, across=across)
    want, tol = ref.norm_rope(x, None, 1e-6, across, None, None, 2.0 ** -8)
    got = qo.cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    ok = ~want.isnan()
    assert ((got - want).abs()[ok] <= tol[ok]).all()


def test_more_rows_than_a_pass_and_far_rows(hsa):
    """More units than the grid holds at once, and a cache past 2^32 elements."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    H, D = 8, 128
    n = sms * 32 * 8 + 100
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn((n, H, D), generator=g, device=DEV).to(torch.bfloat16)
    N = (1 << 32) // (H * D) + n + 5
    kc, vc = (torch.zeros((N, H, D), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    idx = torch.arange(N - 1, N - 1 - n, -1, dtype=torch.int32, device=DEV)
    qo, ko = torch.empty_like(x), torch.empty_like(x)
    for across in (False, True):
        hsa.hsa_qk_norm_rope(x, x, None, None, qo, kc, across=across, v=x, v_out=vc, k_idx=idx)
        for a in range(0, n, n // 5):
            b = min(n, a + n // 5)
            y = torch.empty_like(x[a:b])
            hsa.hsa_qk_norm_rope(x[a:b], x[a:b], None, None, y, ko[a:b], across=across)
            assert torch.equal(y, qo[a:b])
        assert torch.equal(kc[-n:].flip(0), ko) and torch.equal(qo, ko) and torch.equal(vc[-n:].flip(0), x)
        assert not kc[:N - n].any()
    assert hsa.hsa_get_device_error() == 0


def test_same_as_the_rotation_by_itself(hsa):
    """With rows of unit mean square and no weights the call turns as hsa_rope_rows does."""
    n, H, D = 30, 4, 64
    x = (torch.randint(0, 2, (n, H, D), generator=torch.Generator().manual_seed(1)) * 2 - 1).to(torch.bfloat16)
    table = oracle.rope_table((2, 3, 5), D)
    at = torch.arange(n - 1, -1, -1, dtype=torch.int32)
    qo, ko, y = torch.empty_like(x, device=DEV), torch.empty_like(x, device=DEV), x.to(DEV)
    hsa.hsa_qk_norm_rope(x.to(DEV), x.to(DEV), None, None, qo, ko, eps=1e-30, table=table.to(DEV),
                         table_idx=at.to(DEV))
    hsa.hsa_rope_rows(y, at.to(DEV), n, table.to(DEV))
    assert torch.equal(qo, y) and torch.equal(ko, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,Hq,Hkv,D", [(6200, 4, 4, 64), (6200, 4, 1, 64), (6200, 1, 1, 8), (6200, 8, 3, 32),
                                        (6200, 2, 2, 128), (6200, 1, 1, 256), (6200, 32, 32, 8), (3000, 5, 5, 80),
                                        (3000, 12, 3, 96), (3000, 3, 3, 24), (1500, 32, 8, 128), (1500, 40, 40, 128)])
def test_across_heads_token_after_token(hsa, n, Hq, Hkv, D, dtype):
    """More tokens than blocks, so that a block takes several, from one warp a block to as many
    threads as there are; with rows whose squares overflow, and rows of zeros.  The kernel before
    has left NaN where sums are kept."""
    (q, k, v), w, table, at, idx = _inputs(n, Hq, Hkv, D, torch.float32, n + D, True)
    q[5::50] *= 2.0 ** 75
    k[9::31] *= 2.0 ** 90
    k[4::13] = 0.0
    q, k, v = (x.to(dtype) for x in (q, k, v))
    d = [t.to(DEV) for t in (q, k, v, *w, table, at, idx)]
    nan = torch.full((1500, 32, 128), float("nan"), dtype=dtype, device=DEV)
    for rows in (None, d[7]):
        hsa.hsa_qk_norm_rope(nan, nan, None, None, torch.empty_like(nan), torch.empty_like(nan), across=True)
        qo = torch.empty_like(d[0])
        ko, vo = (torch.full((n if rows is None else 2 * n + 3, Hkv, D), 3.0, dtype=dtype, device=DEV) for _ in "kv")
        hsa.hsa_qk_norm_rope(d[0], d[1], d[3], d[4], qo, ko, across=True, table=d[5], table_idx=d[6], v=d[2], v_out=vo,
                             k_idx=rows)
        assert hsa.hsa_get_device_error() == 0
        ko, vo = (x if rows is None else x[rows.long()] for x in (ko, vo))
        for got, x, weight in ((qo, q, w[0]), (ko, k, w[1])):
            _close(got, *ref.norm_rope(x, weight, 1e-6, True, table, at, STEP[dtype]))
        assert torch.equal(vo, d[2])
