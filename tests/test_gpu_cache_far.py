"""The 8-bit cache, paged and packed attention where offsets pass 32 bits: rows near the end
of caches and tensors of more than 4 GiB."""
import numpy as np
import pytest
import torch

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


def test_8_bit_rows_past_4_gib(hsa):
    N, H, D, n = 4_300_000, 16, 64, 37
    kc, vc = (torch.empty((N, H, D), dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.empty((N, H), dtype=torch.uint8, device=DEV) for _ in range(2))
    assert kc.numel() > 2 ** 32
    x = [torch.randn((n, H, D), generator=torch.Generator().manual_seed(s)).to(torch.bfloat16) for s in (1, 2)]
    idx = torch.arange(N - n, N, dtype=torch.int32)
    hsa.hsa_kv_quant_scatter(kc, vc, ks, vs, x[0].to(DEV), x[1].to(DEV), idx.to(DEV), n)
    out = [torch.empty((n, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    hsa.hsa_kv_dequant_gather(kc, vc, ks, vs, idx.to(DEV), n, *out)
    assert hsa.hsa_get_device_error() == 0
    for y, code, scale, got in zip(x, (kc, vc), (ks, vs), out):
        c, s, _ = ref.quantise_rows(y.double().numpy())
        assert torch.equal(code[N - n:].cpu(), torch.from_numpy(c.astype(np.uint8)))
        assert torch.equal(scale[N - n:].cpu(), torch.from_numpy(s))
        assert torch.equal(got.double().cpu(), torch.from_numpy(ref.values(c, s)))


@pytest.mark.parametrize("f8", [False, True])
def test_pages_past_4_gib(hsa, f8):
    page, Hkv, Hq, D, n = 64, 8, 16, 128, 130
    P = (1 << 32) // (page * Hkv * D * (1 if f8 else 2)) + 10
    kind = torch.uint8 if f8 else torch.bfloat16
    kp, vp = (torch.empty((P, page, Hkv, D), dtype=kind, device=DEV) for _ in range(2))
    sc = [torch.empty((P, page, Hkv), dtype=torch.uint8, device=DEV) for _ in range(2)] if f8 else [None, None]
    x = [torch.randn((n, Hkv, D), generator=torch.Generator().manual_seed(s)).to(torch.bfloat16) for s in (3, 4)]
    table = torch.tensor([[P - 1, P - 3, P - 2]], dtype=torch.int32, device=DEV)
    at = torch.arange(n)
    slots = (table[0].cpu().long()[at // page] * page + at % page).int().to(DEV)
    xd = [t.to(DEV) for t in x]
    if f8:
        hsa.hsa_kv_quant_scatter(kp, vp, *sc, *xd, slots, n)
        x = [torch.from_numpy(ref.values(*ref.quantise_rows(t.double().numpy())[:2])) for t in x]
    else:
        hsa.hsa_kv_sync_scatter(kp.view(-1, Hkv, D), vp.view(-1, Hkv, D), *xd, slots, n)
    q = torch.randn((1, 1, Hq, D), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    out = torch.empty((1, 1, Hq, D), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(hsa.hsa_paged_attention_workspace_bytes(1, 1, Hq, Hkv, D), dtype=torch.uint8, device=DEV)
    hsa.hsa_paged_attention(q.to(DEV), kp, vp, table, torch.tensor([n], dtype=torch.int32, device=DEV), out,
                            k_scale=sc[0], v_scale=sc[1], workspace=ws)
    assert hsa.hsa_get_device_error() == 0
    want, tol = ref.attention(q[0].double(), x[0].double(), x[1].double(), [n],
                              p_step=2.0 ** -11 if f8 else 2.0 ** -8)
    assert ((out[0].double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("Hq,D", [(16, 128), (24, 64)])
def test_packed_rows_past_4_gib(hsa, Hq, D):
    """Hq = 24 over 8 K/V heads takes the query rows by the threads, Hq = 16 by TMA."""
    Hkv, n = 8, 150
    T = (1 << 32) // (Hkv * D * 2) + 500
    k, v = (torch.empty((T, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q, out = (torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for t, s in ((q, 6), (k, 7), (v, 8)):
        t[T - n:] = torch.randn((n, *t.shape[1:]), generator=torch.Generator().manual_seed(s)).to(torch.bfloat16)
    cu = torch.tensor([T - n, T], dtype=torch.int32, device=DEV)
    out[T - n - 1] = 9.0
    hsa.hsa_packed_attention(q, k, v, cu, cu, out, mask=1)
    assert hsa.hsa_get_device_error() == 0
    got = out[T - n - 1:].cpu()
    want, tol = ref.attention(*(t[T - n:].double().cpu() for t in (q, k, v)), ref.limits(n, n, 1))
    assert (got[0] == 9.0).all()
    assert ((got[1:].double() - want).abs() <= tol).all()
