"""The 4-bit KV cache on the GPU: what hsa_kv4_quant_scatter writes and hsa_kv4_dequant_gather
reads back, value for value against the 64-bit reference."""
import numpy as np
import pytest
import torch

import oracle
import reference_pages as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def hsa():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2605_06892_gb300 as m
    m.lib()
    torch.cuda.set_device(0)
    m.hsa_get_device_error()
    return m


def _cache(N, H, D, seed):
    """Codes of any kind and words of rows that are written so."""
    g = torch.Generator().manual_seed(seed)
    word = torch.randint(0, 1 << 24, (2, N, H), generator=g) | torch.randint(100, 127, (2, N, H), generator=g) << 24
    return [torch.randint(0, 256, (N, H, D // 2), generator=g).to(torch.uint8) for _ in range(2)] + [
        w.to(torch.int32) for w in word]


def _rows(n, H, D, dtype, seed):
    """Rows of very different sizes, zeros, ties, zero groups and outliers among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, H, D), generator=g)
    x = x * torch.where(torch.rand((1, H, D), generator=g) < 0.05, 20.0, 1.0)
    x = x * torch.exp2(torch.randint(-30, 30, (n, H, 1), generator=g).float())
    x[::5] = torch.randint(-378, 379, x[::5].shape, generator=g).float() / 4   # ties of the codes
    x[1::7, :, torch.from_numpy(ref.group_of(D)) == 2] = 0.0
    x[3::11] = 0.0
    return x.to(dtype)


def _check(hsa, N, H, D, dtype, n, seed, fresh=None):
    host = _cache(N, H, D, seed)
    kf, vf = fresh or (_rows(n, H, D, dtype, seed + 1), _rows(n, H, D, dtype, seed + 2))
    idx = torch.randperm(N, generator=torch.Generator().manual_seed(seed + 3))[:n].int()
    d = [t.to(DEV) for t in host]
    hsa.hsa_kv4_quant_scatter(*d, kf.to(DEV), vf.to(DEV), idx.to(DEV), n)
    bad = False
    others = torch.ones(N, dtype=torch.bool)
    others[idx.long()] = False
    for at, x in ((0, kf), (1, vf)):
        held, words, odd = ref.quantise_rows(x.double().numpy())
        bad |= odd
        code, word = d[at].cpu(), d[2 + at].cpu()
        assert torch.equal(code[others], host[at][others]) and torch.equal(word[others], host[2 + at][others])
        assert np.array_equal(word[idx.long()].numpy().view(np.uint32), words)
        got = ref.values(code[idx.long()].numpy(), words)
        assert np.array_equal(got, held, equal_nan=True)
    assert hsa.hsa_get_device_error() == (-5 if bad else 0)
    return d


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,D,n", [(1, 1, 64, 1), (1, 1, 128, 1), (7, 3, 64, 5), (129, 5, 128, 64),
                                     (300, 12, 64, 131), (40, 7, 128, 40), (3000, 2, 64, 2999)])
def test_written_rows_are_exact(hsa, N, H, D, n, dtype):
    _check(hsa, N, H, D, dtype, n, 100 + N)


@pytest.mark.parametrize("D", [64, 128])
def test_every_border(hsa, D):
    """Each factor 1 .. 63 and each border of the codes: the value, and the next bf16 and the
    next fp32 below and above it."""
    for dtype, bits in ((torch.bfloat16, torch.int16), (torch.float32, torch.int32)):
        rows = []
        for m in range(1, 64):
            for c in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
                t = torch.tensor([m * c], dtype=torch.float32).to(dtype)
                near = torch.cat([(t.view(bits) + d).view(dtype).float() for d in (-1, 0, 1)])
                row = torch.zeros(D)
                run = D // 32
                row[0], row[run] = 6.0 * m, 378.0        # group 0 takes m, group 1 the row's 63
                row[4 * run:4 * run + 3 * 4 * run:4 * run] = near.clamp(max=6.0 * m)
                rows.append(row)
        x = torch.stack(rows)[:, None].to(dtype)
        _check(hsa, len(rows), 1, D, dtype, len(rows), 3, (x, -x * 2.0 ** -20))


def test_edges_of_the_range(hsa):
    """The largest and smallest magnitudes, exact limits of the exponent, signed zeros."""
    f = torch.finfo(torch.float32)
    for dtype in (torch.bfloat16, torch.float32):
        top = torch.finfo(dtype).max
        vals = [378.0, 380.0, 379.0, 1.4765625 * 2 ** 20, 1.4844 * 2 ** 20, top, 252.0 * 2.0 ** 120, f.tiny, f.tiny / 64,
                2.0 ** -100, 2.0 ** -110, 2.0 ** -92, 1.0, -0.0, 6.0 * 2.0 ** -100, 6.03125 * 2.0 ** -100]
        for D in (64, 128):
            x = torch.zeros((len(vals), 1, D))
            for i, a in enumerate(vals):
                x[i, 0, 0] = a
                x[i, 0, 1:9] = torch.tensor([a / 3, -a / 5, -a, a * 0.9375, a / 500, -a / 7000, -0.0, a * 0.53125])
                x[i, 0, 20:24] = a / 63
            x = x.to(dtype)
            _check(hsa, 20, 1, D, dtype, len(vals), 7, (x, -x))


def test_rows_that_are_not_finite(hsa):
    """Held as NaN throughout and reported; read back as NaN, and the rows beside them stay."""
    for dtype in (torch.bfloat16, torch.float32):
        x = _rows(6, 3, 64, dtype, 3)
        y = x.clone()
        x[0, 0, 5] = float("inf")
        x[1, 2, 63] = float("-inf")
        x[2, 1, :] = float("nan")
        x[4, 0, 0], x[4, 0, 1] = float("nan"), torch.finfo(dtype).max
        d = _check(hsa, 9, 3, 64, dtype, 6, 8, (x, y))
        ko, vo = (torch.empty((9, 3, 64), dtype=dtype, device=DEV) for _ in "kv")
        hsa.hsa_kv4_dequant_gather(*d, None, 9, ko, vo)
        nan = ko.isnan()
        assert torch.equal(nan.any(-1), nan.all(-1)) and int(nan.any(-1).sum()) == 4 and not vo.isnan().any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,D,n", [(1, 1, 64, 1), (9, 3, 128, 9), (501, 5, 64, 333), (5000, 3, 128, 4001)])
def test_reading_back(hsa, N, H, D, n, dtype):
    """Rows in any order, the same more than once, all of them, and places without a row."""
    host = _cache(N, H, D, 11)
    d = [t.to(DEV) for t in host]
    k, v = (torch.from_numpy(ref.values(c.numpy(), w.numpy())) for c, w in ((host[0], host[2]), (host[1], host[3])))
    g = torch.Generator().manual_seed(5)
    idx = torch.randint(0, N, (n,), generator=g).int()
    idx[n // 2] = -1
    ko, vo = (torch.full((n + 2, H, D), 7.0, dtype=dtype, device=DEV) for _ in "kv")
    hsa.hsa_kv4_dequant_gather(*d, idx.to(DEV), n, ko, vo)
    for got, want in ((ko, k), (vo, v)):
        want = want[idx.long().clamp(min=0)]
        want[n // 2] = 7.0
        assert torch.equal(got[:n].cpu().double(), want) and (got[n:] == 7).all()
    assert hsa.hsa_get_device_error() == 0
    ko, vo = (torch.full((N, H, D), 7.0, dtype=dtype, device=DEV) for _ in "kv")
    hsa.hsa_kv4_dequant_gather(*d, None, N - 1, ko, vo)
    assert torch.equal(ko[:N - 1].cpu().double(), k[:N - 1]) and (ko[N - 1:] == 7).all()
    assert torch.equal(vo[:N - 1].cpu().double(), v[:N - 1])
    hsa.hsa_kv4_dequant_gather(*d, torch.tensor([N], dtype=torch.int32, device=DEV), 1, ko, vo)
    assert hsa.hsa_get_device_error() == -6


@pytest.mark.parametrize("H,D", [(3, 64), (5, 128)])
def test_rotation_on_the_way(hsa, H, D):
    """The cache holds what the bf16 cache would have held, in 4 bits: fresh rows out of a fused
    projection, into pages, by positions or by the rows themselves; bad and empty places."""
    n, pages, page = 61, 7, 16
    N = pages * page
    g = torch.Generator().manual_seed(2)
    wide = torch.randn((n, 3 * H, D), generator=g).to(torch.bfloat16).to(DEV)
    kf, vf = wide[:, H:2 * H], wide[:, 2 * H:]
    table = oracle.rope_table((4, 5, 6), D)[:N].contiguous().to(DEV)
    idx = torch.randperm(N, generator=g)[:n].int()
    idx[7] = -1
    for at in (None, torch.randint(0, N, (n,), generator=g).int()):
        bad = idx.clone()
        if at is not None:
            at[9] = N + 3                # no such row of the table
        d = [t.view(pages, page, *t.shape[1:]).to(DEV) for t in _cache(N, H, D, 4)]
        before = [t.clone() for t in d]
        hsa.hsa_kv4_quant_scatter(*d, kf, vf, bad.to(DEV), n, table=table,
                                  table_idx=None if at is None else at.to(DEV))
        assert hsa.hsa_get_device_error() == (0 if at is None else -6)
        turned = kf.contiguous()
        rows = idx if at is None else at
        keep = torch.ones(n, dtype=torch.bool)
        keep[7] = False
        if at is not None:
            keep[9] = False
        hsa.hsa_rope_rows(turned, rows.clamp(min=0, max=N - 1).to(DEV), n, table)
        want = [t.clone().flatten(0, 1) for t in before]
        m = int(keep.sum())
        hsa.hsa_kv4_quant_scatter(*want, turned[keep.to(DEV)].contiguous(), vf[keep.to(DEV)].contiguous(),
                                  idx[keep].to(DEV), m)
        assert all(torch.equal(a.flatten(0, 1), b) for a, b in zip(d, want))
        assert hsa.hsa_get_device_error() == 0


def test_many_items_and_far_rows(hsa):
    """More items than a pass of the grid, and rows past 4 GiB of codes."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    H, D = 32, 128
    n = sms * 6 * 256 // 8 // H * 3 + 17
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn((n, H, D), generator=g, device=DEV).to(torch.bfloat16)
    N = (1 << 32) // (H * D // 2) + n + 5
    kc = torch.zeros((N, H, D // 2), dtype=torch.uint8, device=DEV)
    ks = torch.zeros((N, H), dtype=torch.int32, device=DEV)
    vc, vs = kc.clone(), ks.clone()
    idx = torch.arange(N - 1, N - 1 - n, -1, dtype=torch.int32, device=DEV)
    hsa.hsa_kv4_quant_scatter(kc, vc, ks, vs, x, x, idx, n)
    small = [torch.zeros((n, *t.shape[1:]), dtype=t.dtype, device=DEV) for t in (kc, vc, ks, vs)]
    step = n // 7 + 1
    for a in range(0, n, step):          # the same rows in calls of one pass
        b = min(n, a + step)
        part = [t[a:b] for t in small]
        hsa.hsa_kv4_quant_scatter(*part, x[a:b], x[a:b], torch.arange(b - a, dtype=torch.int32, device=DEV), b - a)
    assert torch.equal(kc[-n:].flip(0), small[0]) and torch.equal(ks[-n:].flip(0), small[2])
    assert torch.equal(kc, vc) and torch.equal(ks, vs) and not kc[:-n].any() and not ks[:-n].any()
    out = [torch.empty((n, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    hsa.hsa_kv4_dequant_gather(kc, vc, ks, vs, idx, n, *out[:2])
    hsa.hsa_kv4_dequant_gather(*small, None, n, *out[2:])
    assert all(torch.equal(o, out[0]) for o in out)
    err = (out[0].float() - x.float()).norm() / x.float().norm()
    assert err < 0.125      # half of a step of 1/4 of a value, at most
    assert hsa.hsa_get_device_error() == 0


def test_another_stream_and_graph(hsa):
    """Captured once, replayed on new contents."""
    H, D, n = 4, 64, 50
    d = [t.to(DEV) for t in _cache(80, H, D, 9)]
    eager = [t.clone() for t in d]
    x = _rows(n, H, D, torch.bfloat16, 1).to(DEV)
    idx = torch.arange(n, dtype=torch.int32, device=DEV)
    out = [torch.zeros((n, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        hsa.hsa_kv4_quant_scatter(*d, x, x, idx, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hsa.hsa_kv4_quant_scatter(*d, x, x, idx, n)
        hsa.hsa_kv4_dequant_gather(*d, idx, n, *out[:2])
    x.copy_(_rows(n, H, D, torch.bfloat16, 2))
    idx.copy_(torch.arange(79, 29, -1))
    hsa.hsa_kv4_quant_scatter(*eager, _rows(n, H, D, torch.bfloat16, 1).to(DEV),
                              _rows(n, H, D, torch.bfloat16, 1).to(DEV),
                              torch.arange(n, dtype=torch.int32, device=DEV), n)
    hsa.hsa_kv4_quant_scatter(*eager, x, x, idx, n)
    hsa.hsa_kv4_dequant_gather(*eager, idx, n, *out[2:])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(d, eager))
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    assert hsa.hsa_get_device_error() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_groups_of_very_different_size(hsa, D, dtype):
    """A group far below the row's largest, however far, has a factor of one."""
    group = torch.from_numpy(ref.group_of(D))
    f = torch.finfo(dtype)
    rows = []
    for i, (big, small) in enumerate((b, s) for b in (1e38, f.max, 2.0 ** 100, 1.0, 378.0 * 2.0 ** -100)
                                     for s in (f.tiny, f.tiny / 64, 1e-38, 2.0 ** -60, 2.0 ** -48, 2.0 ** -49, 2.0 ** -50)):
        x = torch.zeros(D)
        x[group == i % 4] = torch.linspace(-big, big, D // 4)
        x[group == (i + 1) % 4] = small
        x[group == (i + 2) % 4] = torch.linspace(-small, small / 3, D // 4)
        rows.append(x)
    x = torch.stack(rows)[:, None].to(dtype)
    assert (x.abs() > 0).any(-1).all()
    _check(hsa, len(rows) + 3, 1, D, dtype, len(rows), 13, (x, -x))
