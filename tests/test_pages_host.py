"""The refusals of the page plan, the normed and rotated rows and the 4-bit cache, without a
GPU: arguments are checked on the host before any launch, and the binding checks what C
cannot see.  And the references of their GPU tests against other ways to the same numbers."""
import ctypes

import numpy as np
import pytest
import torch

import reference_pages as ref

P = ctypes.c_void_p(4096)        # never dereferenced
ODD = ctypes.c_void_p(4104)      # not 16-byte aligned
BYTE = ctypes.c_void_p(4098)     # not 4-byte aligned


@pytest.fixture(scope="module")
def hsa():
    from paper_2605_06892_gb300 import build as b
    b.build()
    import paper_2605_06892_gb300 as m
    m.lib()
    return m


def test_reference_rows():
    """Hand-made rows: codes, factors and exponents worked out on paper."""
    x = np.zeros((1, 64))
    x[0, 0], x[0, 1], x[0, 2], x[0, 63] = 378.0, 31.5, 6.0, -1.0     # groups 0, 0, 1, 3
    held, word, odd = ref.quantise_rows(x)
    assert not odd and word[0] == 127 << 24 | 63 | 1 << 6 | 1 << 18
    # 31.5 / 63 = 0.5; -1 / 1
    assert held[0, 0] == 378.0 and held[0, 1] == 31.5 and held[0, 2] == 6.0 and held[0, 63] == -1.0
    x[0, 0] = 378.5
    assert ref.quantise_rows(x)[1][0] >> 24 == 128
    for v, want in ((2.5, 2.0), (3.5, 4.0), (5.0, 4.0), (0.25, 0.0), (0.75, 1.0), (1.25, 1.0), (1.75, 2.0)):
        x = np.zeros((1, 128))
        x[0, 0], x[0, 3] = 6.0 * 63, 63 * v
        assert ref.quantise_rows(x)[0][0, 3] == 63 * want
    g = np.random.default_rng(1)
    x = g.standard_normal((40, 128)) * np.exp2(g.integers(-20, 20, (40, 1)))
    held, word, _ = ref.quantise_rows(x)
    gr = ref.group_of(128)
    for h in range(4):
        m = word >> (6 * h) & 63
        unit = (m * np.exp2((word >> 24).astype(float) - 127))[:, None]
        # no value lies beyond the largest code, and none is off by more than half a step
        assert (np.abs(x[:, gr == h]) <= 6 * unit).all()
        assert (np.abs(x - held)[:, gr == h] <= unit).all()
    assert (torch.from_numpy(held).to(torch.bfloat16).double().numpy() == held).all()
    codes = np.array([[0x21, 0xf7] + [0] * 30], dtype=np.uint8)     # D = 64
    v = ref.values(codes, np.array([128 << 24 | 3 | 5 << 6], dtype=np.uint32))
    assert list(v[0, :4]) == [0.5 * 3 * 2, 1.0 * 3 * 2, 6.0 * 5 * 2, -6.0 * 5 * 2]


def _quant(hsa, k=P, v=P, ks=P, vs=P, kf=P, kr=None, vf=P, vr=None, idx=P, n=4, N=10, H=2, D=64, dt=0, table=None,
           ids=None, rows=0):
    kr, vr = H * D if kr is None else kr, H * D if vr is None else vr
    return hsa.lib().hsa_kv4_quant_scatter(k, v, ks, vs, kf, kr, vf, vr, idx, n, N, H, D, dt, table, ids, rows, None)


def test_quant_scatter_refusals(hsa):
    c0 = hsa.hsa_launch_count()
    assert _quant(hsa, n=0, k=None, idx=None) == 0
    for bad in (dict(n=-1), dict(N=-1), dict(H=0), dict(D=0), dict(dt=2), dict(dt=3), dict(dt=-1), dict(k=None),
                dict(v=None), dict(ks=None), dict(vs=None), dict(kf=None), dict(vf=None), dict(idx=None),
                dict(k=ODD), dict(v=ODD), dict(kf=ODD), dict(vf=ODD), dict(ks=BYTE), dict(vs=BYTE), dict(ids=P),
                dict(table=P), dict(table=ODD, rows=4), dict(kr=120), dict(kr=132), dict(vr=127), dict(vr=1 << 32),
                dict(kr=-128), dict(kr=0), dict(dt=1, kr=130)):
        assert _quant(hsa, **bad) == -1, bad
    for bad in (dict(D=32), dict(D=96), dict(D=256), dict(n=1 << 30, H=2), dict(H=1 << 25, n=1),
                dict(dt=1, table=P, rows=4)):
        assert _quant(hsa, **bad) == -4, bad
    assert hsa.hsa_launch_count() == c0


def _gather(hsa, k=P, v=P, ks=P, vs=P, idx=P, n=4, N=10, H=2, D=64, ko=P, vo=P, dt=0):
    return hsa.lib().hsa_kv4_dequant_gather(k, v, ks, vs, idx, n, N, H, D, ko, vo, dt, None)


def test_dequant_gather_refusals(hsa):
    c0 = hsa.hsa_launch_count()
    assert _gather(hsa, n=0, k=None) == 0
    for bad in (dict(n=-1), dict(N=-1), dict(H=0), dict(dt=2), dict(k=None), dict(v=None), dict(ks=None),
                dict(vs=None), dict(ko=None), dict(vo=None), dict(k=ODD), dict(ko=ODD), dict(vo=ODD),
                dict(ks=BYTE), dict(vs=BYTE), dict(idx=None, n=11)):
        assert _gather(hsa, **bad) == -1, bad
    for bad in (dict(D=8), dict(D=512), dict(n=1 << 30, H=4)):
        assert _gather(hsa, **bad) == -4, bad
    assert hsa.hsa_launch_count() == c0


def _norm(hsa, q=P, qr=None, k=P, kr=None, v=P, vr=None, qw=P, kw=P, eps=1e-6, across=0, table=P, ids=P, rows=9, n=4,
          Hq=4, Hkv=2, D=64, dt=0, qo=P, ko=P, vo=P, idx=P, N=10):
    qr, kr, vr = (H * D if r is None else r for r, H in ((qr, Hq), (kr, Hkv), (vr, Hkv)))
    return hsa.lib().hsa_qk_norm_rope(q, qr, k, kr, v, vr, qw, kw, eps, across, table, ids, rows, n, Hq, Hkv, D, dt,
                                      qo, ko, vo, idx, N, None)


def test_norm_refusals(hsa):
    c0 = hsa.hsa_launch_count()
    assert _norm(hsa, n=0) == 0
    for bad in (dict(n=-1), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(D=12), dict(D=4), dict(dt=2), dict(dt=3),
                dict(dt=-1), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(v=None), dict(vo=None),
                dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(qo=ODD), dict(ko=ODD), dict(vo=ODD), dict(qw=ODD),
                dict(kw=ODD), dict(table=ODD), dict(table=None), dict(rows=0), dict(N=-1), dict(eps=0.0),
                dict(eps=1e-31), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(qr=248),
                dict(qr=260), dict(kr=120), dict(vr=132), dict(qr=1 << 32), dict(dt=1, qr=258), dict(kr=0)):
        assert _norm(hsa, **bad) == -1, bad
    for bad in (dict(D=264), dict(Hq=1 << 21), dict(Hkv=1 << 21), dict(across=1, Hq=513), dict(across=1, Hkv=513),
                dict(n=2 ** 31 - 1)):
        assert _norm(hsa, **bad) == -4, bad
    assert hsa.hsa_launch_count() == c0


def _plan(hsa, lens=P, want=P, B=3, page=16, table=P, cols=4, free=P, pages=9, nf=P, nfo=P, lo=P, cq=P, slots=P,
          pos=P, new=5, ck=P, rows=P, keys=7):
    return hsa.lib().hsa_page_plan(lens, want, B, page, table, cols, free, pages, nf, nfo, lo, cq, slots, pos, new, ck,
                                   rows, keys, None)


def test_plan_refusals(hsa):
    c0 = hsa.hsa_launch_count()
    for bad in (dict(B=-1), dict(page=0), dict(page=-2), dict(cols=-1), dict(pages=-1), dict(new=-1), dict(keys=-1),
                dict(lens=None), dict(want=None), dict(table=None), dict(free=None), dict(nf=None), dict(nfo=None),
                dict(lo=None), dict(cq=None), dict(slots=None), dict(pos=None), dict(ck=None)):
        assert _plan(hsa, **bad) == -1, bad
    for bad in (dict(page=48), dict(pages=1 << 27), dict(cols=1 << 27), dict(new=2 ** 31 - 1),
                dict(keys=2 ** 31 - 1)):
        assert _plan(hsa, **bad) == -4, bad
    assert hsa.hsa_launch_count() == c0


def test_binding_refuses_what_c_cannot_see(hsa, monkeypatch):
    """Wrong dtypes, shapes, strides and devices, by name and before the library is called."""
    class Lib:
        def __getattr__(self, name):
            def none_called(*a):
                raise AssertionError("reached the library")
            return none_called

    monkeypatch.setattr(hsa, "lib", lambda: Lib())
    u8, i32, bf = torch.uint8, torch.int32, torch.bfloat16
    c, s = torch.zeros((4, 2, 32), dtype=u8), torch.zeros((4, 2), dtype=i32)
    x, i = torch.zeros((3, 2, 64), dtype=bf), torch.zeros(3, dtype=i32)
    with pytest.raises(ValueError, match="CUDA"):
        hsa.hsa_kv4_quant_scatter(c, c, s, s, x, x, i, 3)
    for name, args in (("4 or more rows", (c, c, s, s, x, x, i, 4)), ("v_fresh", (c, c, s, s, x, x[:2], i, 2)),
                       ("v_cache", (c, c[:3], s, s, x, x, i, 2)), ("k_scale", (c, c, s[:3], s, x, x, i, 2)),
                       ("v_scale", (c, c, s, s[:, :1], x, x, i, 2)),
                       ("2 heads x 64", (c, c, s, s, x.view(3, 4, 32), x, i, 3))):
        with pytest.raises(ValueError, match=name):
            hsa.hsa_kv4_quant_scatter(*args)
    with pytest.raises(ValueError, match="table"):
        hsa.hsa_kv4_quant_scatter(c, c, s, s, x, x, i, 2, table=torch.zeros((4, 16, 2)))
    with pytest.raises(TypeError):
        hsa.hsa_kv4_quant_scatter(c.float(), c, s, s, x, x, i, 3)
    with pytest.raises(ValueError, match="v_out"):
        hsa.hsa_kv4_dequant_gather(c, c, s, s, None, 2, x, x[:1])
    with pytest.raises(ValueError, match="4 or more rows"):
        hsa.hsa_kv4_dequant_gather(c, c, s, s, None, 4, x, x)

    q, k, w, t = torch.zeros((3, 4, 64), dtype=bf), x, torch.ones(64), torch.zeros((9, 32, 2))
    ok = dict(q=q, k=k, q_weight=w, k_weight=w, q_out=q, k_out=k)
    for name, change in (("CUDA", {}), ("rows or the head", dict(k=k[:2])), ("rows or the head", dict(k=k[..., :32])),
                         ("q_out", dict(q_out=q[:2])), ("k_out", dict(k_out=k[:2])),
                         ("q_weight", dict(q_weight=w[:32])), ("k_weight", dict(across=True, q_weight=None)),
                         ("table", dict(table=t[:, :16])), ("k_out", dict(k_out=q, k_idx=i)),
                         ("k_idx", dict(k_idx=i[:2])), ("table_idx", dict(table_idx=i[:2])),
                         ("v has", dict(v=k[:2], v_out=k)), ("v_out", dict(v=k, v_out=k[:2]))):
        with pytest.raises(ValueError, match=name):
            hsa.hsa_qk_norm_rope(**{**ok, **change})
    for change in (dict(v=k), dict(v_out=k), dict(q=q.double())):
        with pytest.raises((TypeError, ValueError)):
            hsa.hsa_qk_norm_rope(**{**ok, **change})

    one, lens = torch.zeros(1, dtype=i32), torch.zeros(2, dtype=i32)
    table, cu, new = torch.zeros((2, 4), dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(5, dtype=i32)
    ok = dict(lens=lens, want=lens, page_size=16, page_table=table, free_pages=new, n_free=one, n_free_out=one,
              lens_out=lens, cu_q=cu, slots=new, positions=new)
    for name, change in (("CUDA", {}), ("want", dict(want=cu)), ("lens_out", dict(lens_out=cu)), ("cu_q", dict(cu_q=new)),
                         ("n_free", dict(n_free=lens)), ("n_free_out", dict(n_free_out=lens)),
                         ("page_table", dict(page_table=table[:1])), ("positions", dict(positions=new[:4])),
                         ("cu_k", dict(cu_k=new)), ("more than", dict(page_size=1 << 32))):
        with pytest.raises((ValueError, TypeError), match=name):
            hsa.hsa_page_plan(**{**ok, **change})


def test_attention_over_4_bits_refusals(hsa, monkeypatch):
    def call(q=P, B=2, new=1, Hq=8, k=P, v=P, ks=P, vs=P, pages=10, page=16, Hkv=2, D=64, table=P, cols=4, lens=P,
             out=P, ws=P, size=1 << 30):
        return hsa.lib().hsa_paged_attention(q, B, new, Hq, k, v, ks, vs, pages, page, Hkv, D, 3, table, cols, lens,
                                             0.0, out, ws, size, None)
    c0 = hsa.hsa_launch_count()
    assert call(B=0, q=None, ws=None) == 0 and call(new=0, out=None) == 0
    for bad in (dict(ks=None), dict(vs=None), dict(ks=BYTE), dict(vs=BYTE), dict(k=ODD), dict(v=ODD), dict(Hq=7),
                dict(table=None), dict(lens=None), dict(q=None)):
        assert call(**bad) == -1, bad
    for bad in (dict(D=96), dict(D=32), dict(page=48)):
        assert call(**bad) == -4, bad
    for bad in (dict(ws=None), dict(size=1000)):
        assert call(**bad) == -9, bad
    assert hsa.hsa_launch_count() == c0

    monkeypatch.setattr(hsa, "lib", lambda: None)
    q, t, n = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(
        1, dtype=torch.int32)
    c, w = torch.zeros((2, 16, 2, 32), dtype=torch.uint8), torch.zeros((2, 16, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        hsa.hsa_paged_attention(q, c, c, t, n, q, k_scale=w, v_scale=w)
    monkeypatch.setattr(hsa, "_device", lambda: -1)     # what a tensor of the CPU says
    for name, args in (("head", (torch.zeros((2, 16, 2, 64), dtype=torch.uint8), c, w, w)),
                       ("v_cache", (c, c[:1], w, w)), ("k_scale", (c, c, w[:1], w)), ("v_scale", (c, c, w, w[:1]))):
        with pytest.raises(ValueError, match=name):
            hsa.hsa_paged_attention(q, *args[:2], t, n, q, k_scale=args[2], v_scale=args[3])
    with pytest.raises(TypeError):
        hsa.hsa_paged_attention(q, c, c, t, n, q, k_scale=w)
