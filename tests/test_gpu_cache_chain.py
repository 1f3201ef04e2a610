"""The 8-bit cache, paged and packed attention among the library's other calls, one after
another on one stream: each call may start beside the end of the one before, so what they
hand to one another is compared with the same calls made one at a time."""
import pytest
import torch

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


class Chain:
    """Steps of a server: a prompt's rows go into the caches (bf16 and 8-bit), the layer is
    read back for the active attention, new tokens attend over the pages, and each step's
    results are the next one's inputs."""

    def __init__(self, D, Hq, Hkv):
        g = torch.Generator().manual_seed(7)
        self.P, self.page, self.n, self.B = 24, 16, 90, 3
        self.D, self.Hq, self.Hkv = D, Hq, Hkv
        shape = (self.P, self.page, Hkv, D)

        def new(*s, dtype=torch.bfloat16):
            return torch.randn(s, generator=g).to(dtype).to(DEV)
        self.k8, self.v8 = (torch.zeros(shape, dtype=torch.uint8, device=DEV) for _ in "kv")
        self.ks, self.vs = (torch.full(shape[:3], 127, dtype=torch.uint8, device=DEV) for _ in "kv")
        self.kb, self.vb = (torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        self.back = [torch.zeros((self.P * self.page, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
        self.q = new(self.n, Hq, D)
        self.k, self.v = new(self.n, Hkv, D), new(self.n, Hkv, D)
        self.out = torch.zeros_like(self.q)
        self.small = torch.zeros((self.n, Hkv, D), dtype=torch.bfloat16, device=DEV)
        self.idx = torch.randperm(self.P * self.page, generator=g)[:self.n].int().to(DEV)
        self.table = torch.randperm(self.P, generator=g)[:self.B * 8].view(self.B, 8).int().to(DEV)
        self.lens = torch.tensor([100, 1, 61], dtype=torch.int32, device=DEV)
        self.cu = torch.tensor([0, 31, 31, 90], dtype=torch.int32, device=DEV)
        self.tok = [torch.zeros((self.B, 1, Hq, D), dtype=torch.bfloat16, device=DEV) for _ in "ab"]

    def run(self, hsa, steps, after):
        ws = torch.empty(hsa.hsa_paged_attention_workspace_bytes(3, 1, self.Hq, self.Hkv, self.D),
                         dtype=torch.uint8, device=DEV)
        wp = torch.empty(hsa.hsa_packed_attention_workspace_bytes(self.Hq, self.Hkv, self.D),
                         dtype=torch.uint8, device=DEV)
        flat = (-1, self.Hkv, self.D)
        for i in range(steps):
            calls = (
                lambda: hsa.hsa_packed_attention(self.q, self.k, self.v, self.cu, self.cu, self.out,
                                                 mask=i % 3, workspace=wp),
                lambda: hsa.hsa_kv_quant_scatter(self.k8, self.v8, self.ks, self.vs, self.k, self.v,
                                                 self.idx, self.n),
                lambda: hsa.hsa_kv_sync_scatter(self.kb.view(flat), self.vb.view(flat), self.k, self.v,
                                                self.idx, self.n),
                lambda: hsa.hsa_paged_attention(self.q[:3].view(3, 1, self.Hq, self.D), self.kb, self.vb,
                                                self.table, self.lens, self.tok[0], workspace=ws),
                lambda: hsa.hsa_paged_attention(self.tok[0], self.k8, self.v8, self.table, self.lens,
                                                self.tok[1], k_scale=self.ks, v_scale=self.vs, workspace=ws),
                lambda: hsa.hsa_kv_dequant_gather(self.k8, self.v8, self.ks, self.vs, None,
                                                  self.P * self.page, *self.back),
                lambda: hsa.hsa_active_attention(self.k, None, self.n, *self.back, self.small),
                lambda: hsa.hsa_gather_active(self.tok[1].view(3, -1), torch.arange(
                    2, -1, -1, dtype=torch.int32, device=DEV), 3, self.q[:3].view(3, -1)),
                lambda: hsa.hsa_packed_attention(self.small, self.back[0], self.back[1], self.cu,
                                                 self.cu * 4, self.v, mask=0, workspace=wp),
            )
            for c in calls:
                c()
                after()
        torch.cuda.synchronize()
        return [t.clone() for t in (self.out, self.q, self.v, self.small, *self.tok, self.k8, self.v8, self.ks,
                                    self.vs, self.kb, self.vb, *self.back)]


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 6, 2)])
def test_calls_in_a_row_equal_calls_one_at_a_time(hsa, D, Hq, Hkv):
    alone = Chain(D, Hq, Hkv).run(hsa, 8, torch.cuda.synchronize)
    for _ in range(3):
        row = Chain(D, Hq, Hkv).run(hsa, 8, lambda: None)
        assert all(torch.equal(a, b) for a, b in zip(alone, row))
    assert all(a.float().isfinite().all() for a in alone[:6])
    assert hsa.hsa_get_device_error() == 0


def test_launch_counts(hsa):
    """One launch to write and one to read the 8-bit cache, two for the paged attention, one
    for the packed one, and one more where a cut may follow."""
    c = Chain(64, 4, 2)
    wp = torch.empty(hsa.hsa_packed_attention_workspace_bytes(4, 2, 64), dtype=torch.uint8, device=DEV)
    ws = torch.empty(hsa.hsa_paged_attention_workspace_bytes(3, 1, 4, 2, 64), dtype=torch.uint8, device=DEV)

    def count(f):
        before = hsa.hsa_launch_count()
        f()
        torch.cuda.synchronize()
        return hsa.hsa_launch_count() - before
    assert count(lambda: hsa.hsa_kv_quant_scatter(c.k8, c.v8, c.ks, c.vs, c.k, c.v, c.idx, c.n)) == 1
    assert count(lambda: hsa.hsa_kv_quant_scatter(c.k8, c.v8, c.ks, c.vs, c.k, c.v, c.idx, 0)) == 0
    assert count(lambda: hsa.hsa_kv_dequant_gather(c.k8, c.v8, c.ks, c.vs, None, 9, *c.back)) == 1
    assert count(lambda: hsa.hsa_paged_attention(c.q[:3].view(3, 1, 4, 64), c.kb, c.vb, c.table, c.lens,
                                                 c.tok[0], workspace=ws)) == 2
    assert count(lambda: hsa.hsa_packed_attention(c.q, c.k, c.v, c.cu, c.cu, c.out)) == 1
    assert count(lambda: hsa.hsa_packed_attention(c.q, c.k, c.v, c.cu, c.cu, c.out, workspace=wp)) == 1
    k = torch.zeros((2000, 2, 64), dtype=torch.bfloat16, device=DEV)
    assert count(lambda: hsa.hsa_packed_attention(c.q, k, k, c.cu, c.cu * 20, c.out, workspace=wp)) == 2
    assert hsa.hsa_get_device_error() == 0
