"""Packed attention at the largest number of sequences that it takes."""
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


@pytest.mark.parametrize("Hkv,split", [(1, False), (1, True), (4, False)])
def test_most_sequences(hsa, Hkv, split):
    """All but three of them are empty: blocks pass over the rest while their other warps wait."""
    batch, D, G = (1 << 23) // Hkv, 64, 2
    lens = torch.zeros(batch, dtype=torch.int64)
    at = [0, batch // 2 + 5, batch - 1]
    lens[at] = torch.tensor([300, 170, 301])
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)]).int()
    n = int(cu[-1])
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((n, H, D), generator=g).to(torch.bfloat16) for H in (G * Hkv, Hkv, Hkv))
    out = torch.full((n + 1, G * Hkv, D), 9.0, dtype=torch.bfloat16, device=DEV)
    ws = (torch.empty(hsa.hsa_packed_attention_workspace_bytes(G * Hkv, Hkv, D), dtype=torch.uint8, device=DEV)
          if split else None)
    hsa.hsa_packed_attention(q.to(DEV), k.to(DEV), v.to(DEV), cu.to(DEV), cu.to(DEV), out[:n], mask=1, workspace=ws)
    assert hsa.hsa_get_device_error() == 0
    got = out.cpu()
    assert (got[n] == 9.0).all()
    for b in at:
        i, m = int(cu[b]), int(lens[b])
        want, tol = ref.attention(*(t[i:i + m].double() for t in (q, k, v)), ref.limits(m, m, 1))
        assert ((got[i:i + m].double() - want).abs() <= tol).all()
