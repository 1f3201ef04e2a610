"""Packed attention over values that are not finite: which rows they reach, and that values
which are NaN throughout cost no more than a look."""
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


def _data(n, Hq, Hkv, D, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((n, H, D), generator=g).to(torch.bfloat16) for H in (Hq, Hkv, Hkv)]


def _call(hsa, q, k, v, mask, split=False):
    n, Hq, D = q.shape
    out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device=DEV)
    ws = (torch.empty(hsa.hsa_packed_attention_workspace_bytes(Hq, k.shape[1], D), dtype=torch.uint8, device=DEV)
          if split else None)
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    hsa.hsa_packed_attention(*(t.to(DEV) for t in (q, k, v)), cu, cu, out, mask=mask, workspace=ws)
    assert hsa.hsa_get_device_error() == 0
    return out


def _check(got, q, k, v, mask, rows):
    """An element is NaN (or the infinity that it sees) where its row sees one in that
    dimension, and within the bounds elsewhere."""
    n, Hq, D = q.shape
    Hkv = k.shape[1]
    limit = ref.limits(n, n, mask)[rows]
    finite = torch.where(v.isfinite(), v, torch.zeros_like(v)).double()
    want, tol = ref.attention(q[rows].double(), k.double(), finite, limit)
    odd = ~v.isfinite()
    for i, r in enumerate(rows):
        seen = odd[:int(limit[i])].any(0).repeat_interleave(Hq // Hkv, 0)
        assert not got[r][seen].isfinite().any()
        err = (got[r].double() - want[i]).abs()
        assert (err <= tol[i])[~seen].all(), r


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [1, 90])
@pytest.mark.parametrize("split", [False, True])
def test_rows_see_nan_of_some_dimensions(hsa, split, mask, D):
    """A dimension that is NaN in all keys, and single values behind it: a row that sees NaN in
    the first still has to be formed without the second."""
    n = 2100
    q, k, v = _data(n, 4, 2, D, 1)
    v[:, 0, 3] = float("nan")
    for j, d in ((700, 5), (1500, 40), (2050, D - 1)):
        v[j, 0, d] = float("nan")
    v[1200, 1, 7] = float("inf")
    rows = [0, 1, 89, 90, 640, 698, 699, 700, 1199, 1200, 1300, 1499, 1500, 2000, 2049, 2050, 2099]
    _check(_call(hsa, q, k, v, mask, split).cpu(), q, k, v, mask, rows)


@pytest.mark.parametrize("D", [64, 128])
def test_infinities_of_all_keys(hsa, D):
    """Infinities that a row sees do not make it NaN because of one that it does not see."""
    n = 400
    q, k, v = _data(n, 2, 1, D, 2)
    v[:, 0, 5] = float("inf")
    v[300:, 0, 5] = float("-inf")
    got = _call(hsa, q, k, v, 1).cpu()
    assert (got[:300, :, 5] == float("inf")).all() and got[300:, :, 5].isnan().all()
    _check(got, q, k, v, 1, [0, 100, 255, 299, 300, 399])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [1, 384])
def test_values_that_are_nan_throughout(hsa, mask, D):
    """Such a call takes no longer than a few of the same call over finite values (it took
    hundreds)."""
    n = 20000
    g = torch.Generator(DEV).manual_seed(3)
    q, k, v = (torch.randn((n, H, D), generator=g, device=DEV).to(torch.bfloat16) for H in (4, 2, 2))
    out, cu = torch.empty_like(q), torch.tensor([0, n], dtype=torch.int32, device=DEV)

    def took(values):
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(True), torch.cuda.Event(True)
            a.record()
            hsa.hsa_packed_attention(q, k, values, cu, cu, out, mask=mask)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    usual = took(v)
    assert out.isfinite().all()
    nan = took(torch.full_like(v, float("nan")))
    assert out.isnan().all() and hsa.hsa_get_device_error() == 0
    assert nan < 20 * usual, (usual, nan)
