"""The refusals of the 8-bit cache and the paged attention, without a GPU: arguments are
checked on the host before any launch, and the binding checks what C cannot see."""
import ctypes

import numpy as np
import pytest
import torch

import reference_cache as ref

P = ctypes.c_void_p(4096)        # never dereferenced
ODD = ctypes.c_void_p(4104)      # not 16-byte aligned


@pytest.fixture(scope="module")
def hsa():
    from paper_2605_06892_gb300 import build as b
    b.build()
    import paper_2605_06892_gb300 as m
    m.lib()
    return m


def test_reference_codes_are_torchs():
    """The reference's code table and its rounding against torch's float8_e4m3fn."""
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(ref.VALUES))
    assert np.array_equal(t[~np.isnan(t)], ref.VALUES[~np.isnan(t)])
    x = torch.cat([torch.randn(2000) * 100, torch.arange(-448, 449).float(), torch.arange(-64, 65) / 1024.0])
    x = torch.cat([x.clamp(-448, 448), torch.tensor([448.0])])[None]
    code, scale, odd = ref.quantise_rows(x.double().numpy())
    assert scale.item() == 127 and not odd
    assert np.array_equal(code[0], x[0].to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def _quant(hsa, k=P, v=P, ks=P, vs=P, kf=P, vf=P, idx=P, n=4, N=10, H=2, D=64, dt=0, table=None, ids=None,
           rows=0):
    return hsa.lib().hsa_kv_quant_scatter(k, v, ks, vs, kf, vf, idx, n, N, H, D, dt, table, ids, rows, None)


def test_quant_scatter_refusals(hsa):
    c0 = hsa.hsa_launch_count()
    assert _quant(hsa, n=0, k=None, idx=None) == 0
    for bad in (dict(n=-1), dict(N=-1), dict(H=0), dict(D=0), dict(D=12), dict(dt=2), dict(dt=-1), dict(k=None),
                dict(v=None), dict(ks=None), dict(vs=None), dict(kf=None), dict(vf=None), dict(idx=None),
                dict(k=ODD), dict(v=ODD), dict(kf=ODD), dict(vf=ODD), dict(ids=P), dict(table=P),
                dict(table=ODD, rows=4)):
        assert _quant(hsa, **bad) == -1, bad
    for bad in (dict(D=264), dict(n=1 << 30, H=2), dict(dt=1, table=P, rows=4)):
        assert _quant(hsa, **bad) == -4, bad
    assert hsa.hsa_launch_count() == c0


def _gather(hsa, k=P, v=P, ks=P, vs=P, idx=P, n=4, N=10, H=2, D=64, ko=P, vo=P, dt=0):
    return hsa.lib().hsa_kv_dequant_gather(k, v, ks, vs, idx, n, N, H, D, ko, vo, dt, None)


def test_dequant_gather_refusals(hsa):
    c0 = hsa.hsa_launch_count()
    assert _gather(hsa, n=0, k=None) == 0
    for bad in (dict(n=-1), dict(N=-1), dict(H=0), dict(D=4), dict(D=20), dict(dt=2), dict(k=None), dict(v=None),
                dict(ks=None), dict(vs=None), dict(ko=None), dict(vo=None), dict(k=ODD), dict(ko=ODD),
                dict(vo=ODD), dict(idx=None, n=11)):
        assert _gather(hsa, **bad) == -1, bad
    for bad in (dict(D=512), dict(n=1 << 30, H=4)):
        assert _gather(hsa, **bad) == -4, bad
    assert hsa.hsa_launch_count() == c0


def _paged(hsa, q=P, B=2, new=1, Hq=8, k=P, v=P, ks=None, vs=None, pages=10, page=16, Hkv=2, D=64, dt=0, table=P,
           cols=4, lens=P, out=P, ws=P, size=1 << 30):
    return hsa.lib().hsa_paged_attention(q, B, new, Hq, k, v, ks, vs, pages, page, Hkv, D, dt, table, cols, lens,
                                         0.0, out, ws, size, None)


def test_paged_attention_refusals(hsa):
    c0 = hsa.hsa_launch_count()
    assert _paged(hsa, B=0, q=None, ws=None) == 0 and _paged(hsa, new=0, out=None) == 0
    for bad in (dict(B=-1), dict(new=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=7), dict(pages=-1), dict(cols=-1),
                dict(page=0), dict(dt=3), dict(q=None), dict(out=None), dict(lens=None), dict(k=None),
                dict(v=None), dict(table=None), dict(q=ODD), dict(out=ODD), dict(k=ODD), dict(v=ODD),
                dict(dt=2), dict(dt=2, ks=P)):
        assert _paged(hsa, **bad) == -1, bad
    for bad in (dict(dt=1), dict(D=96), dict(page=48), dict(pages=1 << 27), dict(cols=1 << 27),
                dict(Hq=65538, Hkv=2), dict(B=1 << 20, new=1 << 10)):
        assert _paged(hsa, **bad) == -4, bad
    for bad in (dict(ws=None), dict(ws=ODD), dict(size=1000)):
        assert _paged(hsa, **bad) == -9, bad
    assert hsa.hsa_launch_count() == c0


def test_workspace_sizes(hsa):
    size = hsa.hsa_paged_attention_workspace_bytes
    assert size(1, 1, 8, 2, 64) > 0 and size(1, 1, 8, 2, 64) == size(64, 4, 12, 12, 64)
    assert size(1, 1, 8, 2, 128) > size(1, 1, 8, 2, 64)
    for none in ((0, 1, 8, 2, 64), (1, 0, 8, 2, 64), (1, 1, 7, 2, 64), (1, 1, 8, 2, 96)):
        assert size(*none) == 0


def test_binding_refuses_what_c_cannot_see(hsa, monkeypatch):
    """Wrong dtypes, shapes, strides and devices, before the library is called."""
    def none_called(*a):
        raise AssertionError("reached the library")

    class Lib:
        hsa_kv_quant_scatter = hsa_kv_dequant_gather = hsa_paged_attention = staticmethod(none_called)

    monkeypatch.setattr(hsa, "lib", lambda: Lib)
    c, s = torch.zeros((4, 2, 64), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8)
    x, i = torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        hsa.hsa_kv_quant_scatter(c, c, s, s, x, x, i, 3)
    with pytest.raises(ValueError, match="4 or more rows"):
        hsa.hsa_kv_quant_scatter(c, c, s, s, x, x, i, 4)
    with pytest.raises(ValueError, match="rows of 2 heads x 64"):
        hsa.hsa_kv_quant_scatter(c, c, s, s, x.view(3, 4, 32), x, i, 3)
    with pytest.raises(TypeError):
        hsa.hsa_kv_quant_scatter(c.float(), c, s, s, x, x, i, 3)
    with pytest.raises(ValueError, match="4 or more rows"):
        hsa.hsa_kv_dequant_gather(c, c, s, s, None, 4, x, x)
    with pytest.raises(ValueError, match="CUDA"):
        hsa.hsa_kv_dequant_gather(c, c, s, s, i, 3, x, x)
    q = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16)
    pages = torch.zeros((2, 16, 2, 64), dtype=torch.bfloat16)
    t, n = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        hsa.hsa_paged_attention(q, pages, pages, t, n, q)
    with pytest.raises(TypeError):
        hsa.hsa_paged_attention(q.float(), pages, pages, t, n, q)


def _packed(hsa, q=P, qr=512, k=P, kr=128, v=P, vr=128, cq=P, ck=P, B=2, tq=10, tk=10, Hq=8, Hkv=2, D=64, mask=1,
            out=P, dt=0, ws=None, size=0):
    return hsa.lib().hsa_packed_attention(q, qr, k, kr, v, vr, cq, ck, B, tq, tk, Hq, Hkv, D, mask, 0.0, out, dt,
                                          ws, size, None)


def test_packed_attention_refusals(hsa):
    c0 = hsa.hsa_launch_count()
    assert _packed(hsa, B=0, q=None) == 0 and _packed(hsa, tq=0, q=None, out=None) == 0
    for bad in (dict(B=-1), dict(tq=-1), dict(tk=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=7), dict(mask=-1),
                dict(dt=2), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(cq=None),
                dict(ck=None), dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(out=ODD), dict(qr=504),
                dict(qr=516), dict(kr=120), dict(kr=132), dict(vr=64), dict(vr=1 << 32)):
        assert _packed(hsa, **bad) == -1, bad
    for bad in (dict(dt=1), dict(D=96, qr=768, kr=192, vr=192), dict(tk=2 ** 31 - 1), dict(tq=1 << 30),
                dict(Hq=1 << 19, qr=1 << 25)):
        assert _packed(hsa, **bad) == -4, bad
    for bad in (dict(ws=ODD, size=1 << 30), dict(ws=P, size=1000)):
        assert _packed(hsa, **bad) == -9, bad
    assert hsa.hsa_launch_count() == c0
    size = hsa.hsa_packed_attention_workspace_bytes
    assert size(8, 2, 128) > size(8, 2, 64) > 0 and size(8, 3, 64) == 0 and size(8, 2, 96) == 0


def test_packed_binding_refuses_what_c_cannot_see(hsa, monkeypatch):
    monkeypatch.setattr(hsa, "lib", lambda: None)
    q, k = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros((4, 1, 64), dtype=torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        hsa.hsa_packed_attention(q, k, k, cu, cu, q)
    with pytest.raises(TypeError):
        hsa.hsa_packed_attention(q.float(), k, k, cu, cu, q)
    with pytest.raises(ValueError, match="lie together"):
        hsa.hsa_packed_attention(torch.zeros((4, 64, 2), dtype=torch.bfloat16).transpose(1, 2), k, k, cu, cu, q)


def test_binding_names_what_is_wrong(hsa, monkeypatch):
    """Shapes that do not go together are refused by name."""
    monkeypatch.setattr(hsa, "lib", lambda: None)
    c, s = torch.zeros((4, 2, 64), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8)
    x, i = torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for name, args in (("v_fresh", (c, c, s, s, x, x[:2], i, 2)), ("v_cache", (c, c[:3], s, s, x, x, i, 2)),
                       ("k_scale", (c, c, s[:3], s, x, x, i, 2)), ("v_scale", (c, c, s, s[:, :1], x, x, i, 2))):
        with pytest.raises(ValueError, match=name):
            hsa.hsa_kv_quant_scatter(*args)
    with pytest.raises(ValueError, match="table"):
        hsa.hsa_kv_quant_scatter(c, c, s, s, x, x, i, 2, table=torch.zeros((4, 16, 2)))
    with pytest.raises(ValueError, match="v_out"):
        hsa.hsa_kv_dequant_gather(c, c, s, s, None, 2, x, x[:1])
    q, pages = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 16, 2, 64), dtype=torch.bfloat16)
    t, n = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="batch"):
        hsa.hsa_paged_attention(q, pages, pages, t, n.repeat(2), q)
    with pytest.raises(ValueError, match="out"):
        hsa.hsa_paged_attention(q, pages, pages, t, n, q[:, :, :2])
    k, cu = torch.zeros((4, 1, 64), dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32)
    p = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    for name, args in (("v has", (p, k, k[:3], cu, cu, p)), ("cu_k", (p, k, k, cu, cu[:1], p)),
                       ("out", (p, k, k, cu, cu, p[:3])), ("head", (p, k[:, :, :32], k, cu, cu, p))):
        with pytest.raises(ValueError, match=name):
            hsa.hsa_packed_attention(*args)
