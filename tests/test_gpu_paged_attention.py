"""Attention of the newest tokens over paged caches, bf16 and 8-bit, against the 64-bit
reference: group sizes, lengths from none to several runs, pages that end inside a tile,
unread rows that hold NaN, and what the call reports."""
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


class Pool:
    """Pages with sequences of the given lengths in shuffled pages; every row that no
    sequence owns holds NaN."""

    def __init__(self, lens, page, Hkv, D, f8, seed, spread=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.f8 = lens, f8
        need = [-(-n // page) for n in lens]
        P = sum(need) + 2
        order = torch.randperm(P, generator=g).tolist()
        cols = max(max(need), 1)
        self.table = torch.full((len(lens), cols), -7, dtype=torch.int32)   # past the end: never read
        self.k, self.v = (torch.full((P, page, Hkv, D), float("nan")) for _ in range(2))
        if f8:
            self.k, self.v = (torch.full((P, page, Hkv, D), 0x7f, dtype=torch.uint8) for _ in range(2))
            self.ks, self.vs = (torch.full((P, page, Hkv), 255, dtype=torch.uint8) for _ in range(2))
        self.keys = []
        for b, n in enumerate(lens):
            pages = [order.pop() for _ in range(need[b])]
            self.table[b, :need[b]] = torch.tensor(pages, dtype=torch.int32)
            at = torch.tensor([pages[j // page] for j in range(n)], dtype=torch.long), torch.arange(n) % page
            kv = []
            for name in ("k", "v"):
                x = torch.randn((n, Hkv, D), generator=g)
                if spread:
                    x = x * torch.exp2(torch.randint(-spread, spread + 1, (n, Hkv, 1), generator=g).float())
                x = x.to(torch.bfloat16)
                if f8:
                    c, s, _ = ref.quantise_rows(x.double().numpy()) if n else (np.zeros((0, Hkv, D)), np.zeros((0, Hkv)), 0)
                    getattr(self, name)[at] = torch.from_numpy(c.astype(np.uint8))
                    getattr(self, name + "s")[at] = torch.from_numpy(s.astype(np.uint8))
                    x = torch.from_numpy(ref.values(c, s))
                else:
                    getattr(self, name)[at] = x.float()
                kv.append(x.double())
            self.keys.append(kv)
        if not f8:
            self.k, self.v = self.k.to(torch.bfloat16), self.v.to(torch.bfloat16)

    def call(self, hsa, q, out, ws, scale=0.0, **kw):
        d = dict(k_scale=self.ks.to(DEV), v_scale=self.vs.to(DEV)) if self.f8 else {}
        hsa.hsa_paged_attention(q, self.k.to(DEV), self.v.to(DEV), self.table.to(DEV),
                                torch.tensor(self.lens, dtype=torch.int32, device=DEV), out,
                                scale=scale, workspace=ws, **d, **kw)


def _ws(hsa, B, n, Hq, Hkv, D):
    return torch.empty(hsa.hsa_paged_attention_workspace_bytes(B, n, Hq, Hkv, D), dtype=torch.uint8, device=DEV)


def _check(hsa, lens, new, Hq, Hkv, D, page, f8, seed, spread=0, scale=0.0, qsize=1.0):
    pool = Pool(lens, page, Hkv, D, f8, seed, spread)
    B = len(lens)
    q = (torch.randn((B, new, Hq, D), generator=torch.Generator().manual_seed(seed + 1)) * qsize).to(torch.bfloat16)
    out = torch.full((B + 1, new, Hq, D), 9.0, dtype=torch.bfloat16, device=DEV)
    pool.call(hsa, q.to(DEV), out[:B], _ws(hsa, B, new, Hq, Hkv, D), scale)
    assert hsa.hsa_get_device_error() == 0
    got = out.double().cpu()
    assert (got[B] == 9.0).all()
    for b, n in enumerate(lens):
        k, v = pool.keys[b]
        want, tol = ref.attention(q[b].double(), k, v, ref.limits(new, n, 1), scale or None,
                                  p_step=2.0 ** -11 if f8 else 2.0 ** -8)
        err = (got[b] - want).abs()
        assert (err <= tol).all(), (b, n, float((err / tol).max()))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[1], [0, 5, 0], [15, 16, 17, 33], [63, 64, 65, 127, 128, 129, 200]])
def test_short_lengths(hsa, lens, D, f8):
    _check(hsa, lens, 1, 8, 2, D, 16, f8, 1 + sum(lens))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (12, 12), (10, 2), (32, 2), (40, 2), (7, 7)])
def test_groups(hsa, Hq, Hkv, f8):
    _check(hsa, [90, 301], 1, Hq, Hkv, 64, 32, f8, Hq)
    _check(hsa, [90, 301], 1, Hq, Hkv, 128, 32, f8, Hq + 100)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("new", [2, 3, 5, 17])
def test_several_new_tokens_are_causal(hsa, new, f8):
    _check(hsa, [new, 1, 0, 64, 130, 400], new, 8, 4, 64, 8, f8, new)
    _check(hsa, [new, 2, 129], new, 6, 2, 128, 8, f8, new + 50)


@pytest.mark.parametrize("page", [1, 2, 8, 256, 4096])
def test_page_sizes(hsa, page):
    for f8 in (False, True):
        _check(hsa, [77, 300, 3], 1, 4, 2, 128, page, f8, page)


@pytest.mark.parametrize("f8", [False, True])
def test_long_sequences_are_split_and_joined(hsa, f8):
    """Far more tiles than blocks, units that span many blocks, and a block that holds the
    end of one unit, whole units and the start of another."""
    _check(hsa, [30011], 1, 4, 1, 128, 64, f8, 3)
    _check(hsa, [9000, 40, 12000, 0, 1, 130], 2, 4, 2, 64, 16, f8, 4)


@pytest.mark.parametrize("f8", [False, True])
def test_many_sequences(hsa, f8):
    """More sequences than threads of a block, so that a thread counts several."""
    lens = [(37 * b) % 150 for b in range(600)]
    _check(hsa, lens, 1, 2, 1, 64, 16, f8, 5)


@pytest.mark.parametrize("f8", [False, True])
def test_scales_of_very_different_size(hsa, f8):
    """Rows of K and V from 2^-20 to 2^20, so that the largest contribution is not the
    largest score's, and scores of hundreds."""
    _check(hsa, [40, 700], 1, 8, 2, 64, 16, f8, 6, spread=20, scale=2.0 ** -22)
    _check(hsa, [513], 2, 4, 2, 128, 16, f8, 7, spread=3, qsize=8.0)


@pytest.mark.parametrize("f8", [False, True])
def test_explicit_scale(hsa, f8):
    _check(hsa, [100], 1, 4, 2, 64, 16, f8, 8, scale=0.3)


@pytest.mark.parametrize("f8", [False, True])
def test_nan_of_a_newer_token_stays_with_the_rows_that_see_it(hsa, f8):
    D, new, Hq, Hkv = 64, 4, 8, 2
    for n, at in ((100, 98), (130, 127), (128, 125)):
        pool = Pool([n], 16, Hkv, D, f8, 11)
        j = int(pool.table[0, at // 16]), at % 16
        pool.v[j[0], j[1], 1, 3] = 0x7f if f8 else float("nan")
        pool.k[j[0], j[1], 1, 7] = 0x7f if f8 else float("nan")
        q = torch.randn((1, new, Hq, D), generator=torch.Generator().manual_seed(12)).to(torch.bfloat16)
        out = torch.empty((1, new, Hq, D), dtype=torch.bfloat16, device=DEV)
        pool.call(hsa, q.to(DEV), out, _ws(hsa, 1, new, Hq, Hkv, D))
        got = out[0].double().cpu()
        k, v = pool.keys[0]
        want, tol = ref.attention(q[0].double(), k, v, ref.limits(new, n, 1), p_step=2.0 ** -8)
        clean = torch.ones((new, Hq), dtype=torch.bool)
        clean[at - (n - new):, Hq // 2:] = False
        assert ((got - want).abs()[clean] <= tol[clean]).all()
        assert got[~clean].isnan().all()
    assert hsa.hsa_get_device_error() == 0


def test_bad_pages_and_lengths_are_reported(hsa):
    D, Hq, Hkv = 64, 4, 2
    pool = Pool([40, 20], 16, Hkv, D, False, 13)
    q = torch.randn((2, 1, Hq, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    ws = _ws(hsa, 2, 1, Hq, Hkv, D)
    out = torch.empty((2, 1, Hq, D), dtype=torch.bfloat16, device=DEV)
    good = pool.table.clone()
    for bad in (-1, pool.k.shape[0], 2 ** 31 - 1):
        pool.table = good.clone()
        pool.table[0, 1] = bad
        pool.call(hsa, q.to(DEV), out, ws)
        assert hsa.hsa_get_device_error() == -6
        # the page reads as rows of zeros
        k, v = (t.clone() for t in pool.keys[0])
        k[16:32], v[16:32] = 0.0, 0.0
        want, tol = ref.attention(q[0].double(), k, v, [40])
        assert ((out[0].double().cpu() - want).abs() <= tol).all()
    pool.table = good
    pool.lens = [-5, 20]
    pool.call(hsa, q.to(DEV), out, ws)
    assert hsa.hsa_get_device_error() == -6
    assert (out[0] == 0).all()
    pool.table = good[:, :2].contiguous()      # room for 32 keys
    pool.lens = [40, 20]
    pool.call(hsa, q.to(DEV), out, ws)
    assert hsa.hsa_get_device_error() == -6
    want, tol = ref.attention(q[0].double(), pool.keys[0][0][:32], pool.keys[0][1][:32], [32])
    assert ((out[0].double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("f8", [False, True])
def test_captured_steps_follow_the_lengths(hsa, f8):
    """A captured step replayed while the sequences grow, on a stream of its own: each step
    writes the new token's K/V into its slot and attends."""
    D, Hq, Hkv, page = 64, 8, 2, 16
    start = [30, 64]
    pool = Pool([n + 3 for n in start], page, Hkv, D, f8, 14)
    dev = dict(k=pool.k.to(DEV), v=pool.v.to(DEV), table=pool.table.to(DEV))
    if f8:
        dev |= dict(ks=pool.ks.to(DEV), vs=pool.vs.to(DEV))
    lens = torch.tensor(start, dtype=torch.int32, device=DEV)
    slot = torch.zeros(2, dtype=torch.int32, device=DEV)
    fresh = [torch.zeros((2, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    q = torch.zeros((2, 1, Hq, D), dtype=torch.bfloat16, device=DEV)
    out = torch.empty_like(q)
    ws = _ws(hsa, 2, 1, Hq, Hkv, D)

    def one():
        if f8:
            hsa.hsa_kv_quant_scatter(dev["k"], dev["v"], dev["ks"], dev["vs"], *fresh, slot, 2)
        else:
            hsa.hsa_kv_sync_scatter(dev["k"].view(-1, Hkv, D), dev["v"].view(-1, Hkv, D), *fresh, slot, 2)
        lens.add_(1)
        hsa.hsa_paged_attention(q, dev["k"], dev["v"], dev["table"], lens, out, k_scale=dev.get("ks"),
                                v_scale=dev.get("vs"), workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        slot.copy_(torch.tensor([int(pool.table[b, start[b] // page]) * page + start[b] % page for b in range(2)]))
        with torch.cuda.graph(graph, stream=side):
            one()
        g = torch.Generator().manual_seed(15)
        kv = [[t[:n].clone() for t in pool.keys[b]] for b, n in enumerate(start)]
        for step in range(3):
            at = [n + step for n in start]
            slot.copy_(torch.tensor([int(pool.table[b, at[b] // page]) * page + at[b] % page for b in range(2)]))
            x = [torch.randn((2, Hkv, D), generator=g).to(torch.bfloat16) for _ in range(2)]
            for t, y in zip(fresh, x):
                t.copy_(y)
            qn = torch.randn((2, 1, Hq, D), generator=g).to(torch.bfloat16)
            q.copy_(qn)
            graph.replay()
            side.synchronize()
            for b in range(2):
                for i in range(2):
                    y = x[i][b:b + 1].double()
                    if f8:
                        y = torch.from_numpy(ref.values(*ref.quantise_rows(y.numpy())[:2]))
                    kv[b][i] = torch.cat([kv[b][i], y])
                want, tol = ref.attention(qn[b].double(), *kv[b], [at[b] + 1],
                                          p_step=2.0 ** -11 if f8 else 2.0 ** -8)
                assert ((out[b].double().cpu() - want).abs() <= tol).all()
    assert hsa.hsa_get_device_error() == 0


def test_same_result_in_any_company(hsa):
    """A call's result has the same bits alone and beside another stream's calls."""
    pool = Pool([5000, 77], 32, 2, 128, False, 16)
    q = torch.randn((2, 1, 8, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    outs = [torch.empty_like(q) for _ in range(3)]
    wss = [_ws(hsa, 2, 1, 8, 2, 128) for _ in range(2)]
    pool.call(hsa, q, outs[0], wss[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            pool.call(hsa, q, outs[1 + i], wss[i])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,new", [(17, 1), (31, 1), (33, 1), (8, 5), (3, 23)])
def test_many_rows_per_head(hsa, Hq, new, D, f8):
    """More than 16 rows of one K/V head, also more than a unit takes, over units of several
    tiles, cut ones among them."""
    _check(hsa, [2000, 129, new, 0, 40], new, Hq, 1, D, 32, f8, Hq + D)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_nan_among_many_rows(hsa, D, f8):
    """As above with a value that is not finite among the newest keys."""
    new, Hq, n, at = 9, 4, 300, 296
    pool = Pool([n], 16, 1, D, f8, 31)
    j = int(pool.table[0, at // 16]), at % 16
    pool.v[j[0], j[1], 0, 3] = 0x7f if f8 else float("inf")
    q = torch.randn((1, new, Hq, D), generator=torch.Generator().manual_seed(32)).to(torch.bfloat16)
    out = torch.empty((1, new, Hq, D), dtype=torch.bfloat16, device=DEV)
    pool.call(hsa, q.to(DEV), out, _ws(hsa, 1, new, Hq, 1, D))
    got = out[0].double().cpu()
    want, tol = ref.attention(q[0].double(), *pool.keys[0], ref.limits(new, n, 1))
    blind = at - (n - new)
    assert ((got - want).abs()[:blind] <= tol[:blind]).all()
    assert not got[blind:, :, 3].isfinite().any()
    clean = [d for d in range(D) if d != 3]
    assert ((got - want).abs()[blind:, :, clean] <= tol[blind:, :, clean]).all()
    assert hsa.hsa_get_device_error() == 0


def test_values_over_the_whole_range(hsa):
    """8-bit values of one sequence from 2^-100 to 2^100: the weights of keys whose values
    are tiny count in the sum all the same, zeros among them."""
    D, n, Hq = 64, 96, 4
    pool = Pool([n], 16, 1, D, True, 41)
    g = torch.Generator().manual_seed(42)
    v = torch.randn((n, 1, D), generator=g) * torch.exp2((torch.arange(n) % 3 * 100.0 - 100.0))[:, None, None]
    v[::7] = 0.0
    code, scale, _ = ref.quantise_rows(v.to(torch.bfloat16).double().numpy())
    at = torch.tensor([int(pool.table[0, j // 16]) for j in range(n)]), torch.arange(n) % 16
    pool.v[at], pool.vs[at] = torch.from_numpy(code.astype(np.uint8)), torch.from_numpy(scale)
    held = torch.from_numpy(ref.values(code, scale))
    ws = _ws(hsa, 1, 1, Hq, 1, D)
    q = torch.randn((1, 1, Hq, D), generator=g).to(torch.bfloat16)
    out = torch.empty((1, 1, Hq, D), dtype=torch.bfloat16, device=DEV)
    pool.call(hsa, q.to(DEV), out, ws)
    want, tol = ref.attention(q[0].double(), pool.keys[0][0], held, [n], p_step=2.0 ** -11)
    assert ((out[0].double().cpu() - want).abs() <= tol).all()
    assert hsa.hsa_get_device_error() == 0
