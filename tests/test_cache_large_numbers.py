"""Numbers that C's int does not hold are refused by the binding: passed on, their low 32 bits
would be another call's."""
import pytest
import torch


@pytest.fixture(scope="module")
def hsa():
    from paper_2605_06892_gb300 import build as b
    b.build()
    import paper_2605_06892_gb300 as m
    m.lib()
    return m


def _no_library(hsa, monkeypatch):
    """Places every tensor and fails where the library would be called."""
    monkeypatch.setattr(hsa, "lib", lambda: pytest.fail("reached the library"))
    monkeypatch.setattr(hsa, "_place", lambda name, t, dtype, device: 0)


@pytest.mark.parametrize("mask", [2 ** 32 + 1, 2 ** 31, 1 - 2 ** 32])
def test_mask(hsa, monkeypatch, mask):
    _no_library(hsa, monkeypatch)
    x, cu = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError, match="mask"):
        hsa.hsa_packed_attention(x, x, x, cu, cu, x, mask=mask)


def test_rows_of_the_cache_and_of_the_call(hsa, monkeypatch):
    _no_library(hsa, monkeypatch)
    n = 2 ** 32 + 3
    big = torch.zeros((1, 1, 8), dtype=torch.uint8).expand(n, 1, 8)
    small = torch.zeros((4, 1, 8), dtype=torch.uint8)
    rows = torch.zeros((1, 1, 8), dtype=torch.bfloat16)
    idx = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="k_cache"):
        hsa.hsa_kv_quant_scatter(big, big, big[..., 0], big[..., 0], rows.expand(4, 1, 8), rows.expand(4, 1, 8), idx, 3)
    with pytest.raises(ValueError, match="k_out"):
        hsa.hsa_kv_dequant_gather(small, small, small[..., 0], small[..., 0], idx[:1].expand(n), n,
                                  rows.expand(n, 1, 8), rows.expand(n, 1, 8))
    with pytest.raises(ValueError, match="k_fresh"):
        hsa.hsa_kv_quant_scatter(small, small, small[..., 0], small[..., 0], rows.expand(n, 1, 8),
                                 rows.expand(n, 1, 8), idx[:1].expand(n), n)
