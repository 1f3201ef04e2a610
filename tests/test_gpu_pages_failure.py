"""Waits that run out in the 4-bit paged attention and in the norm across heads: through the test
hook a first load never comes; the call reports HSA_ERR_TIMEOUT, ends soon, and the same context
then runs a normal call to the right result."""
import time

import pytest
import torch

import reference_pages as ref
import test_gpu_paged4 as paged

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


def _stalled(hsa, call):
    assert hsa.hsa_test_inject_attention_stall(1) == 0
    try:
        t0 = time.time()
        call()
        status = hsa.hsa_get_device_error()
        assert time.time() - t0 < 30
    finally:
        hsa.hsa_test_inject_attention_stall(0)
    assert status == -7


@pytest.mark.parametrize("D,page,lens,new,Hq", [(64, 16, [700, 3, 64], 1, 4), (128, 1, [300, 129], 2, 12),
                                                (128, 128, [40, 5000], 1, 8)])
def test_paged_attention(hsa, D, page, lens, new, Hq):
    pool = paged.Pool(paged._random(lens, 2, D, 3), page, 2, D, 3)
    q = paged._normal((len(lens), new, Hq, D), 4).to(torch.bfloat16)
    ws = paged._ws(hsa, len(lens), new, Hq, 2, D)
    out = torch.empty_like(q, device=DEV)
    _stalled(hsa, lambda: pool.call(hsa, q.to(DEV), out, ws))
    pool.call(hsa, q.to(DEV), out, ws)
    assert hsa.hsa_get_device_error() == 0
    for b in range(len(lens)):
        want, tol = pool.want(b, q[b], new)
        assert ((out[b].double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("n", [400, 3000])
def test_norm_across_heads(hsa, n):
    H, D = 6, 64
    g = torch.Generator().manual_seed(2)
    x = torch.randn((n, H, D), generator=g).to(torch.bfloat16)
    angle = torch.randn((n, D // 2), generator=g)
    table = torch.stack([angle.cos(), angle.sin()], -1)
    qo, ko = (torch.empty((n, H, D), dtype=torch.bfloat16, device=DEV) for _ in "qk")

    def call():
        hsa.hsa_qk_norm_rope(x.to(DEV), x.to(DEV), None, None, qo, ko, across=True, table=table.to(DEV))
    _stalled(hsa, call)
    call()
    assert hsa.hsa_get_device_error() == 0
    want, tol = ref.norm_rope(x, None, 1e-6, True, table, torch.arange(n), 2.0 ** -8)
    assert ((qo.double().cpu() - want).abs() <= tol).all() and torch.equal(qo, ko)
