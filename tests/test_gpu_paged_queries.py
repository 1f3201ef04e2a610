"""4-bit paged attention whose query rows come from far and whose keys are near: every unit's rows
are there before they are read."""
import numpy as np
import pytest
import torch

import reference_cache as base
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


@pytest.mark.parametrize("new,Hq,Hkv,D", [(1, 8, 2, 128), (1, 12, 12, 64), (4, 8, 2, 128), (5, 4, 2, 64)])
def test_queries_in_memory_and_pages_in_cache(hsa, new, Hq, Hkv, D):
    """Thousands of short sequences over the same few pages, the queries' lines out of L2: the
    same bits as with all of them in L2, and the reference's values."""
    B, page, P = 3000, 16, 12
    g = torch.Generator().manual_seed(Hq + D)
    x = torch.randn((2, P * page, Hkv, D), generator=g).to(torch.bfloat16).double().numpy()
    pair, word, _ = ref.encode_rows(x)
    held = torch.from_numpy(ref.values(pair, word))
    codes = [torch.from_numpy(c).view(P, page, Hkv, D // 2).to(DEV) for c in pair]
    words = [torch.from_numpy(w.view(np.int32)).view(P, page, Hkv).to(DEV) for w in word]
    table = torch.stack([torch.randperm(P, generator=g) for _ in range(B)]).int()
    lens = torch.randint(0, P * page + 1, (B,), generator=g).int()
    q = torch.randn((B, new, Hq, D), generator=g).to(torch.bfloat16)
    d = [t.to(DEV) for t in (q, table, lens)]
    out = torch.empty_like(d[0])
    ws = torch.empty(hsa.hsa_paged_attention_workspace_bytes(B, new, Hq, Hkv, D), dtype=torch.uint8, device=DEV)

    def call():
        out.fill_(9.0)
        hsa.hsa_paged_attention(d[0], *codes, d[1], d[2], out, k_scale=words[0], v_scale=words[1], workspace=ws)
        return out.clone()
    call()
    near = call()
    other = torch.empty(1 << 29, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        other.fill_(1)                     # more than L2 holds
        for t in (*codes, *words, d[1]):
            t.sum()
        assert torch.equal(call(), near)
    assert hsa.hsa_get_device_error() == 0
    for b in range(0, B, 500):
        n = int(lens[b])
        at = (table[b].long()[torch.arange(n) // page] * page + torch.arange(n) % page)
        k, v = held[0][at], held[1][at]
        limit = base.limits(new, n, 1)
        want, tol = base.attention(q[b].double(), k, v, limit, p_step=ref.P_STEP)
        tol = tol + ref.small_weights(q[b].double(), k, torch.from_numpy(word[1].view(np.int32))[at].numpy(), limit)
        assert ((near[b].double().cpu() - want).abs() <= tol).all()
