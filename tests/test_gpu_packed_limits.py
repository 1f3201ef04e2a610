"""Packed attention at the largest number of sequences and the largest scores that it takes."""
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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask,split", [(0, False), (1, False), (1, True)])
@pytest.mark.parametrize("most", [2.0 ** 12, 2.0 ** 25, 2.0 ** 29.9])
def test_largest_score_takes_all(hsa, most, mask, split, D):
    """Scores of up to just below 2^30.  The largest that a row sees is further from the next than
    the sums' rounding, so that its output is that key's value: off by the output's rounding,
    and by 2^-8 for the one probability's, whose unrounded value divides it, and 2^-20."""
    lq, n, Hq = 40, 2000, 2
    g = torch.Generator().manual_seed(2)
    k, v = torch.randn((n, 1, D), generator=g), torch.randn((n, 1, D), generator=g).to(torch.bfloat16)
    q = torch.randn((lq, Hq, D), generator=g).to(torch.bfloat16)
    k = k.to(torch.bfloat16)
    limit = torch.from_numpy(ref.limits(lq, n, mask))
    s = torch.einsum("ihd,jd->ihj", q.double(), k[:, 0].double())
    scale = most / s.abs().max().item()
    s = (s * scale).masked_fill(torch.arange(n) >= limit[:, None, None], -torch.inf)
    top, at = s.topk(2, dim=-1)
    apart = torch.einsum("ihd,jd->ihj", q.double().abs(), k[:, 0].double().abs()).amax() * scale * (D + 2) * 2.0 ** -23
    sure = top[..., 0] - top[..., 1] > apart + 40
    assert sure.double().mean() > 0.5   # rows that the test can tell
    out = torch.full((lq, Hq, D), 9.0, dtype=torch.bfloat16, device=DEV)
    ws = (torch.empty(hsa.hsa_packed_attention_workspace_bytes(Hq, 1, D), dtype=torch.uint8, device=DEV)
          if split else None)
    cu = [torch.tensor([0, m], dtype=torch.int32, device=DEV) for m in (lq, n)]
    hsa.hsa_packed_attention(q.to(DEV), k.to(DEV), v.to(DEV), *cu, out, mask=mask, scale=scale, workspace=ws)
    assert hsa.hsa_get_device_error() == 0
    want = v[at[..., 0], 0].double()
    err = (out.cpu().double() - want).abs()
    assert (err <= (2.0 ** -7 + 2.0 ** -20) * want.abs())[sure].all()
