"""The 8-bit KV cache on the GPU: what hsa_kv_quant_scatter writes and
hsa_kv_dequant_gather reads back, bit for bit against the 64-bit reference."""
import numpy as np
import pytest
import torch

import oracle
import reference_cache as ref

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
    g = torch.Generator().manual_seed(seed)
    return ([torch.randint(0, 0x7f, (N, H, D), generator=g).to(torch.uint8) for _ in range(2)] +
            [torch.randint(100, 150, (N, H), generator=g).to(torch.uint8) for _ in range(2)])


def _rows(n, H, D, dtype, seed):
    """Rows of very different sizes, zeros and ties among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, H, D), generator=g)
    x = x * torch.exp2(torch.randint(-30, 30, (n, H, 1), generator=g).float())
    x[::5] = torch.randint(-32, 33, x[::5].shape, generator=g).float() / 2   # ties of the codes
    x[3::11] = 0.0
    return x.to(dtype)


def _check(hsa, N, H, D, dtype, n, seed, fresh=None):
    kc, vc, ks, vs = _cache(N, H, D, seed)
    kf, vf = fresh or (_rows(n, H, D, dtype, seed + 1), _rows(n, H, D, dtype, seed + 2))
    idx = torch.randperm(N, generator=torch.Generator().manual_seed(seed + 3))[:n].int()
    d = [t.to(DEV) for t in (kc, vc, ks, vs)]
    hsa.hsa_kv_quant_scatter(d[0].view(torch.float8_e4m3fn), d[1].view(torch.float8_e4m3fn), d[2], d[3],
                             kf.to(DEV), vf.to(DEV), idx.to(DEV), n)
    bad = False
    for code, scale, x in ((kc, ks, kf), (vc, vs, vf)):
        c, s, odd = ref.quantise_rows(x.double().numpy())
        code[idx.long()], scale[idx.long()] = torch.from_numpy(c.astype(np.uint8)), torch.from_numpy(s)
        bad |= odd
    for got, want in zip(d, (kc, vc, ks, vs)):
        got = got.cpu()
        if got.dim() == 3:   # a NaN may have either sign
            got, want = (torch.where(t & 0x7f == 0x7f, torch.full_like(t, 0x7f), t) for t in (got, want))
        assert torch.equal(got, want)
    assert hsa.hsa_get_device_error() == (-5 if bad else 0)
    return d


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,D,n", [(1, 1, 8, 1), (7, 3, 16, 5), (129, 5, 64, 64), (300, 12, 128, 131),
                                     (40, 7, 96, 40), (33, 2, 256, 9), (64, 4, 40, 64), (5000, 4, 64, 4999)])
def test_written_codes_are_exact(hsa, N, H, D, n, dtype):
    _check(hsa, N, H, D, dtype, n, 100 + N)


def test_many_items_take_more_than_one_pass(hsa):
    """More (token, head) items than the grid holds at once: 32 blocks of 256 threads on
    each SM, two items of 8 lanes each."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    H, D = 16, 8
    n = sms * 32 * 256 * 2 // H + 1000
    g = torch.Generator().manual_seed(5)
    x = torch.randint(-448, 449, (n, H, D), generator=g).to(torch.bfloat16)
    kc = torch.zeros((n, H, D), dtype=torch.uint8, device=DEV)
    ks = torch.zeros((n, H), dtype=torch.uint8, device=DEV)
    vc, vs = kc.clone(), ks.clone()
    idx = torch.arange(n - 1, -1, -1, dtype=torch.int32, device=DEV)
    xd = x.to(DEV)
    hsa.hsa_kv_quant_scatter(kc, vc, ks, vs, xd, xd, idx, n)
    a = xd.float().abs().amax(-1)
    e = torch.ceil(torch.log2(a / 448)).clamp(min=-100)   # exact here: a is a small integer
    e = torch.where(a == 0, torch.full_like(e, -100.0), e)
    want = (xd.float() * torch.exp2(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(kc.flip(0), want) and torch.equal(vc, kc)
    assert torch.equal(ks.flip(0), (e + 127).to(torch.uint8)) and torch.equal(vs, ks)
    ko = torch.empty((n, H, D), dtype=torch.bfloat16, device=DEV)
    vo = torch.empty_like(ko)
    hsa.hsa_kv_dequant_gather(kc, vc, ks, vs, idx, n, ko, vo)
    back = (want.view(torch.float8_e4m3fn).float() * torch.exp2(e)[..., None]).to(torch.bfloat16)
    assert torch.equal(ko, back) and torch.equal(vo, back)


def test_edges_of_the_range(hsa):
    """The largest and smallest magnitudes, exact limits of the scale, signed zeros."""
    f = torch.finfo(torch.float32)
    for dtype in (torch.bfloat16, torch.float32):
        top = torch.finfo(dtype).max
        vals = [448.0, 449.0, 464.0, 1.75 * 2 ** 20, 1.7501 * 2 ** 20, top, 1.875 * 2.0 ** 127, f.tiny,
                f.tiny / 64, 2.0 ** -100, 2.0 ** -110, 2.0 ** -92, 1.0, -0.0]
        x = torch.zeros((len(vals), 1, 32))
        for i, a in enumerate(vals):
            x[i, 0, 0] = a
            x[i, 0, 1:9] = torch.tensor([a / 3, -a / 5, -a, a * 0.9375, a / 500, -a / 7000, -0.0, a * 0.53125])
        x = x.to(dtype)
        _check(hsa, 20, 1, 32, dtype, len(vals), 7, (x, -x))


def test_non_finite_elements_become_nan_and_are_reported(hsa):
    for dtype in (torch.bfloat16, torch.float32):
        x = _rows(6, 3, 64, dtype, 3)
        y = x.clone()
        x[0, 0, 5] = float("inf")
        x[1, 2, 63] = float("-inf")
        x[2, 1, :] = float("nan")
        x[4, 0, 0] = float("nan")
        x[4, 0, 1] = torch.finfo(dtype).max
        d = _check(hsa, 9, 3, 64, dtype, 6, 8, (x, y))
        assert int((d[0] & 0x7f == 0x7f).sum()) >= 67
        ko = torch.empty((9, 3, 64), dtype=dtype, device=DEV)
        vo = torch.empty_like(ko)
        hsa.hsa_kv_dequant_gather(d[0], d[1], d[2], d[3], None, 9, ko, vo)
        assert torch.equal(ko.isnan(), d[0] & 0x7f == 0x7f) and not vo.isnan().any()
        assert hsa.hsa_get_device_error() == 0


@pytest.mark.parametrize("D,H", [(64, 5), (128, 3), (96, 2)])
def test_rotated_keys_equal_the_bf16_cache_in_8_bits(hsa, D, H):
    """With a table the cache holds what hsa_kv_sync_scatter_rope would have written,
    quantised, whether the table's rows go by idx or by their own indices."""
    grid, n = (3, 7, 9), 100
    N = 3 * 7 * 9
    table = oracle.rope_table(grid, D).to(DEV)
    kf, vf = (_rows(n, H, D, torch.bfloat16, s).clamp(-1e4, 1e4).to(DEV) for s in (21, 22))
    idx = torch.randperm(N, generator=torch.Generator().manual_seed(4))[:n].int().to(DEV)
    kc, vc = (torch.zeros((N, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    hsa.hsa_kv_sync_scatter_rope(kc, vc, kf, vf, idx, n, table)
    want = [ref.quantise_rows(t.double().cpu().numpy()) for t in (kc, vc)]
    for own_rows in (False, True):
        slots = torch.randperm(N, generator=torch.Generator().manual_seed(5))[:n].int().to(DEV)
        at = slots if own_rows else idx
        d = [t.to(DEV) for t in _cache(N, H, D, 6)]
        hsa.hsa_kv_quant_scatter(d[0], d[1], d[2], d[3], kf, vf, at, n, table=table,
                                 table_idx=idx if own_rows else None)
        src = idx.long().cpu()
        for code, scale, (c, s, _) in zip(d[:2], d[2:], want):
            got = code[at.long()].cpu()
            assert torch.equal(got, torch.from_numpy(c.astype(np.uint8))[src])
            assert torch.equal(scale[at.long()].cpu(), torch.from_numpy(s)[src])
    assert hsa.hsa_get_device_error() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,H,N,n", [(64, 3, 50, 31), (128, 12, 300, 300), (8, 1, 4, 1), (96, 5, 77, 20)])
def test_rows_read_back_are_exact(hsa, D, H, N, n, dtype):
    kc, vc, ks, vs = _cache(N, H, D, 30 + D)
    kc[0, 0, :4] = torch.tensor([0x80, 0x81, 0xff, 0x01], dtype=torch.uint8)
    ks[0, 0], ks[1, 0], vs[0, 0] = 27, 247, 247
    kc[1] %= 0x78   # below 2^128 at the largest scale
    vc[0] %= 0x78
    d = [t.to(DEV) for t in (kc, vc, ks, vs)]
    idx = torch.randint(0, N, (n,), generator=torch.Generator().manual_seed(9)).int()
    for at in (idx, None):
        ko, vo = (torch.full((n + 1, H, D), 7.0, dtype=dtype, device=DEV) for _ in range(2))
        hsa.hsa_kv_dequant_gather(*d, None if at is None else at.to(DEV), n, ko, vo)
        src = torch.arange(n) if at is None else at.long()
        for got, code, scale in ((ko, kc, ks), (vo, vc, vs)):
            want = torch.from_numpy(ref.values(code[src].numpy(), scale[src].numpy()))
            assert torch.equal(got[:n].double().cpu().nan_to_num(5.0), want.nan_to_num(5.0))
            assert torch.equal(got[:n].isnan().cpu(), want.isnan())
            assert (got[n] == 7.0).all()
    assert hsa.hsa_get_device_error() == 0


def test_bad_indices_skip_their_rows(hsa):
    N, H, D, n = 20, 2, 64, 6
    kc, vc, ks, vs = (t.to(DEV) for t in _cache(N, H, D, 1))
    before = [t.clone() for t in (kc, vc, ks, vs)]
    x = _rows(n, H, D, torch.bfloat16, 2).to(DEV)
    idx = torch.tensor([3, -1, 5, N, 2 ** 31 - 1, 0], dtype=torch.int32, device=DEV)
    hsa.hsa_kv_quant_scatter(kc, vc, ks, vs, x, x, idx, n)
    assert hsa.hsa_get_device_error() == -6
    keep = torch.ones(N, dtype=torch.bool)
    keep[[3, 5, 0]] = False
    for got, was in zip((kc, vc, ks, vs), before):
        assert torch.equal(got[keep.to(DEV)], was[keep.to(DEV)])
    out = torch.full((n, H, D), 3.0, dtype=torch.bfloat16, device=DEV)
    out2 = out.clone()
    hsa.hsa_kv_dequant_gather(kc, vc, ks, vs, idx, n, out, out2)
    assert hsa.hsa_get_device_error() == -6
    assert (out[[1, 3, 4]] == 3.0).all() and (out2[[1, 3, 4]] == 3.0).all()
    # a table row out of range
    table = torch.zeros((4, D // 2, 2), device=DEV)
    was = [t.clone() for t in (kc, vc, ks, vs)]
    ids = torch.tensor([4, -1], dtype=torch.int32, device=DEV)
    hsa.hsa_kv_quant_scatter(kc, vc, ks, vs, x, x, torch.tensor([1, 2], dtype=torch.int32, device=DEV), 2,
                             table=table, table_idx=ids)
    assert hsa.hsa_get_device_error() == -6
    assert all(torch.equal(a, b) for a, b in zip((kc, vc, ks, vs), was))


def test_layer_with_an_8_bit_cache_in_a_graph(hsa):
    """One iteration of a layer as it is used: active rows into the 8-bit cache, the layer
    read back into a shared bf16 buffer, the active attention over it; captured and
    replayed on new rows, on a stream of its own."""
    N, H, D, n = 500, 4, 64, 130
    kc, vc, ks, vs = (t.to(DEV) for t in _cache(N, H, D, 40))
    table = oracle.rope_table((5, 10, 10), D).to(DEV)
    idx = torch.randperm(N, generator=torch.Generator().manual_seed(2))[:n].sort().values.int().to(DEV)
    x = [_rows(n, H, D, torch.bfloat16, s).clamp(-3, 3).to(DEV) for s in (1, 2)]
    q = torch.randn((n, H, D), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    kb, vb = (torch.empty((N, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    out = torch.empty_like(q)
    ws = torch.empty(hsa.hsa_active_attention_workspace_bytes(n, N, H, D), dtype=torch.uint8, device=DEV)

    def layer():
        hsa.hsa_kv_quant_scatter(kc, vc, ks, vs, x[0], x[1], idx, n, table=table)
        hsa.hsa_kv_dequant_gather(kc, vc, ks, vs, None, N, kb, vb)
        hsa.hsa_active_attention(q, None, n, kb, vb, out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer()
        for s in (50, 51):
            for t, seed in zip(x, (s, s + 10)):
                t.copy_(_rows(n, H, D, torch.bfloat16, seed).clamp(-3, 3))
            graph.replay()
            side.synchronize()
            k8 = torch.from_numpy(ref.values(kc.cpu().numpy(), ks.cpu().numpy()))
            v8 = torch.from_numpy(ref.values(vc.cpu().numpy(), vs.cpu().numpy()))
            assert torch.equal(kb.double().cpu(), k8) and torch.equal(vb.double().cpu(), v8)
            want, tol = ref.attention(q.double().cpu(), k8, v8, [N] * n)
            assert ((out.double().cpu() - want).abs() <= tol).all()
            rot = x[0].clone()
            hsa.hsa_rope_rows(rot, idx, n, table)
            c, sc, _ = ref.quantise_rows(rot.double().cpu().numpy())
            assert torch.equal(kc[idx.long()].cpu(), torch.from_numpy(c.astype(np.uint8)))
            assert torch.equal(ks[idx.long()].cpu(), torch.from_numpy(sc))
    assert hsa.hsa_get_device_error() == 0
