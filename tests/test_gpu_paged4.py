"""Attention of the newest tokens over 4-bit caches in pages, against the 64-bit reference over
the values that the codes stand for: group sizes, lengths from none to several runs, pages that
end inside a tile, unread rows that hold NaN, rows of NaN, sizes of values and scores, and what
the call reports."""
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


def _held(x):
    """Codes, words and the values that they stand for, of rows x [n, Hkv, D]."""
    pair, word, _ = ref.encode_rows(x.to(torch.bfloat16).double().numpy())
    return torch.from_numpy(pair), torch.from_numpy(word.view(np.int32)), torch.from_numpy(ref.values(pair, word))


class Pool:
    """Pages with sequences of the given lengths in shuffled pages; every row that no sequence
    owns holds NaN, and every entry of the table that names none is out of range."""

    def __init__(self, kv, page, Hkv, D, seed):
        g = torch.Generator().manual_seed(seed)
        self.lens = [k.shape[0] for k, _ in kv]
        need = [-(-n // page) for n in self.lens]
        P = sum(need) + 2
        order = torch.randperm(P, generator=g).tolist()
        self.table = torch.full((len(kv), max(max(need), 1)), -7, dtype=torch.int32)
        self.codes = [torch.randint(0, 256, (P, page, Hkv, D // 2), generator=g).to(torch.uint8) for _ in "kv"]
        self.words = [torch.full((P, page, Hkv), -1, dtype=torch.int32) for _ in "kv"]     # s = 255
        self.held, self.v_words = [], []
        for b, pair in enumerate(kv):
            n = self.lens[b]
            pages = [order.pop() for _ in range(need[b])]
            self.table[b, :need[b]] = torch.tensor(pages, dtype=torch.int32)
            at = torch.tensor([pages[j // page] for j in range(n)], dtype=torch.long), torch.arange(n) % page
            rows = []
            for i, x in enumerate(pair):
                c, w, y = _held(x)
                self.codes[i][at], self.words[i][at] = c, w
                rows.append(y)
            self.held.append(rows)
            self.v_words.append(w)

    def call(self, hsa, q, out, ws, scale=0.0, **kw):
        hsa.hsa_paged_attention(q, *(t.to(DEV) for t in self.codes), self.table.to(DEV),
                                torch.tensor(self.lens, dtype=torch.int32, device=DEV), out,
                                k_scale=self.words[0].to(DEV), v_scale=self.words[1].to(DEV), scale=scale,
                                workspace=ws, **kw)

    def want(self, b, q, new, scale=None):
        """(out, tolerance) of sequence b's rows q [new, Hq, D]."""
        limit = base.limits(new, self.lens[b], 1)
        want, tol = base.attention(q.double(), *self.held[b], limit, scale, p_step=ref.P_STEP)
        return want, tol + ref.small_weights(q.double(), self.held[b][0], self.v_words[b], limit, scale)


def _normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def _random(lens, Hkv, D, seed, spread=0):
    g = torch.Generator().manual_seed(seed)
    kv = []
    for n in lens:
        x = torch.randn((2, n, Hkv, D), generator=g)
        x[0] *= torch.where(torch.rand((1, Hkv, D), generator=g) < 0.05, 4.0, 1.0)
        if spread:
            x = x * torch.exp2(torch.randint(-spread, spread + 1, (2, n, Hkv, 1), generator=g).float())
        kv.append((x[0], x[1]))
    return kv


def _ws(hsa, B, n, Hq, Hkv, D):
    return torch.empty(hsa.hsa_paged_attention_workspace_bytes(B, n, Hq, Hkv, D), dtype=torch.uint8, device=DEV)


def _compare(hsa, kv, q, page, scale=None, seed=0):
    B, new, Hq, D = q.shape
    Hkv = kv[0][0].shape[1]
    pool = Pool(kv, page, Hkv, D, seed)
    out = torch.full((B + 1, new, Hq, D), 9.0, dtype=torch.bfloat16, device=DEV)
    pool.call(hsa, q.to(DEV), out[:B], _ws(hsa, B, new, Hq, Hkv, D), scale or 0.0)
    assert hsa.hsa_get_device_error() == 0
    got = out.double().cpu()
    assert (got[B] == 9.0).all()
    for b in range(B):
        want, tol = pool.want(b, q[b], new, scale)
        err = (got[b] - want).abs()
        assert (err <= tol).all(), (b, pool.lens[b], float((err / tol).max()))


def _check(hsa, lens, new, Hq, Hkv, D, page, seed, spread=0, scale=None, qsize=1.0):
    q = (_normal((len(lens), new, Hq, D), seed + 1) * qsize).to(torch.bfloat16)
    _compare(hsa, _random(lens, Hkv, D, seed, spread), q, page, scale, seed)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[1], [0, 5, 0], [15, 16, 17, 33], [63, 64, 65, 127, 128, 129, 200]])
def test_short_lengths(hsa, lens, D):
    _check(hsa, lens, 1, 8, 2, D, 16, 1 + sum(lens))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (12, 12), (10, 2), (32, 2), (40, 2), (7, 7)])
def test_groups(hsa, Hq, Hkv, D):
    _check(hsa, [90, 301], 1, Hq, Hkv, D, 32, Hq + D)


@pytest.mark.parametrize("new", [2, 3, 5, 17])
def test_several_new_tokens_are_causal(hsa, new):
    _check(hsa, [new, 1, 0, 64, 130, 400], new, 8, 4, 64, 8, new)
    _check(hsa, [new, 2, 129], new, 6, 2, 128, 8, new + 50)


@pytest.mark.parametrize("page", [1, 2, 8, 256, 4096])
def test_page_sizes(hsa, page):
    _check(hsa, [77, 300, 3], 1, 4, 2, 128, page, page)
    _check(hsa, [77, 300, 3], 2, 4, 2, 64, page, page)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [4, 16, 32, 64, 128])
def test_ends_of_tiles(hsa, page, D):
    """Lengths about the ends of what a warp and a block hold, pages that end inside."""
    lens = [47, 49, 191, 192, 193, 223, 225, 255, 256, 257, 289, 321, 511, 512, 513]
    _check(hsa, lens, 1, 4, 2, D, page, 60 + page)
    _check(hsa, [n + 2 for n in lens], 3, 2, 2, D, page, 61 + page)


def test_two_graphs_that_share_a_workspace(hsa):
    """Captured with different batches and row counts over one workspace, replayed in turn."""
    calls = []
    ws = torch.empty(max(hsa.hsa_paged_attention_workspace_bytes(2, 1, 8, 2, 128),
                         hsa.hsa_paged_attention_workspace_bytes(3, 5, 4, 2, 64)), dtype=torch.uint8, device=DEV)
    for lens, new, Hq, D in (([3000, 700], 1, 8, 128), ([5, 900, 4000], 5, 4, 64)):
        pool = Pool(_random(lens, 2, D, 70 + D), 32, 2, D, 70 + D)
        q = _normal((len(lens), new, Hq, D), 71).to(torch.bfloat16)
        d = [t.to(DEV) for t in (q, *pool.codes, pool.table, torch.tensor(lens, dtype=torch.int32))]
        words = [t.to(DEV) for t in pool.words]
        out, graph = torch.empty_like(d[0]), torch.cuda.CUDAGraph()

        def run():
            hsa.hsa_paged_attention(*d, out, k_scale=words[0], v_scale=words[1], workspace=ws)
        run()
        first = out.clone()
        for b in range(len(lens)):
            want, tol = pool.want(b, q[b], new)
            assert ((out[b].double().cpu() - want).abs() <= tol).all()
        with torch.cuda.graph(graph):
            run()
        calls.append((graph, out, first, d, words))
    for _ in range(3):
        for _, out, *_ in calls:
            out.fill_(9.0)
        for graph, *_ in calls:
            graph.replay()
        assert all(torch.equal(out, first) for _, out, first, *_ in calls)
    assert hsa.hsa_get_device_error() == 0


def test_long_sequences_are_split_and_joined(hsa):
    _check(hsa, [30011], 1, 4, 1, 128, 64, 3)
    _check(hsa, [9000, 40, 12000, 0, 1, 130], 2, 4, 2, 64, 16, 4)


def test_many_sequences(hsa):
    _check(hsa, [(37 * b) % 150 for b in range(600)], 1, 2, 1, 64, 16, 5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,new", [(17, 1), (31, 1), (33, 1), (8, 5), (3, 23)])
def test_many_rows_per_head(hsa, Hq, new, D):
    _check(hsa, [2000, 129, new, 0, 40], new, Hq, 1, D, 32, Hq + D)


def test_sizes_of_values(hsa):
    """Rows of K and V from 2^-20 to 2^20, so that the largest contribution is not the largest
    score's, and scores of hundreds; a scale of one's own."""
    _check(hsa, [40, 700], 1, 8, 2, 64, 16, 6, spread=20, scale=2.0 ** -22)
    _check(hsa, [513], 2, 4, 2, 128, 16, 7, spread=3, qsize=8.0)
    _check(hsa, [100], 1, 4, 2, 64, 16, 8, scale=0.3)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ek,eq", [(110, -112), (118, -100), (-98, 112), (100, 20), (-90, -30)])
def test_keys_and_queries_of_very_different_size(hsa, ek, eq, D):
    n = 200
    k, v = _normal((n, 2, D), 11) * 2.0 ** ek, _normal((n, 2, D), 12)
    k[5], k[77] = 0.0, 0.0
    q = (_normal((1, 2, 4, D), 13) * 2.0 ** eq).to(torch.bfloat16)
    _compare(hsa, [(k, v)], q, 128, scale=D ** -0.5 * 2.0 ** -(ek + eq))


@pytest.mark.parametrize("new,Hq", [(1, 4), (2, 12)])
@pytest.mark.parametrize("D,zeros", [(128, 140000), (64, 280000)])
def test_long_stretch_of_zero_rows(hsa, D, zeros, new, Hq):
    """More zero rows than 32 bits count at their power of two's inverse, then 100 others."""
    page, P = 128, -(-(zeros + 100) // 128)
    k, v = torch.zeros((zeros + 100, 1, D)), torch.zeros((zeros + 100, 1, D))
    k[zeros:], v[zeros:] = _normal((100, 1, D), 1), _normal((100, 1, D), 2)
    q = _normal((1, new, Hq, D), 3).to(torch.bfloat16)
    for least in (0, 27 << 24):          # words as fresh memory holds them, and as they are written
        codes = [torch.zeros((P * page, 1, D // 2), dtype=torch.uint8) for _ in "kv"]
        words = [torch.full((P * page, 1), least, dtype=torch.int32) for _ in "kv"]
        held = []
        for i, x in enumerate((k, v)):
            codes[i][zeros:zeros + 100], words[i][zeros:zeros + 100], y = _held(x[zeros:])
            held.append(torch.cat([torch.zeros((zeros, 1, D), dtype=torch.float64), y]))
        out = torch.empty((1, new, Hq, D), dtype=torch.bfloat16, device=DEV)
        hsa.hsa_paged_attention(
            q.to(DEV), *(c.view(P, page, 1, -1).to(DEV) for c in codes),
            torch.arange(P, dtype=torch.int32, device=DEV)[None],
            torch.tensor([zeros + 100], dtype=torch.int32, device=DEV), out,
            k_scale=words[0].view(P, page, 1).to(DEV), v_scale=words[1].view(P, page, 1).to(DEV),
            workspace=_ws(hsa, 1, new, Hq, 1, D))
        assert hsa.hsa_get_device_error() == 0
        limit = base.limits(new, zeros + 100, 1)
        want, tol = base.attention(q[0].double(), *held, limit, p_step=ref.P_STEP)
        tol = tol + ref.small_weights(q[0].double(), held[0], words[1], limit)
        assert want.abs().amax() > 0 and ((out[0].double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("D", [64, 128])
def test_small_weights_count_at_the_top_of_the_range(hsa, D):
    """Values up to 2^127: 60000 keys whose weights are about 2^-20 of one key's weigh a few per
    cent together."""
    n = 60001
    k = torch.zeros((n, 1, D))
    k[1:, 0, 0], k[0, 0, 0] = -16.0, 4.0
    q = torch.zeros((1, 1, 2, D))
    q[..., 0] = 1.0
    v = (torch.rand((n, 1, D), generator=torch.Generator().manual_seed(10)) * 0.5 + 0.5) * 2.0 ** 127
    _compare(hsa, [(k, v)], q.to(torch.bfloat16), 128, scale=0.6931471805599453)


@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_climb(hsa, D):
    """Each tile's scores are far above all before them, then far below, while the values'
    sizes go the other way."""
    n = 3000
    up = torch.arange(n) < 2000
    level = torch.where(up, torch.arange(n) * 0.25, 500.0 - (torch.arange(n) - 2000) * 0.5)
    k = _normal((n, 1, D), 14) * 0.05
    k[:, 0, 0] = level
    q = _normal((1, 1, 4, D), 15)
    q[..., 0] = torch.tensor([1.0, 0.25, -1.0, 0.0])
    v = _normal((n, 1, D), 16) * torch.exp2(-level / 8)[:, None, None]
    _compare(hsa, [(k, v)], q.to(torch.bfloat16), 128, scale=0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", [10, 20, 25, 26, 31, 60, 100])
def test_scores_of_any_size(hsa, D, sign, power):
    """Scores are small numbers times 2^power, exactly, so that the keys that share the largest
    have all the weight, in equal parts, whatever their values' sizes: off by the rounding of
    probabilities and output, by 2^-20 for the exponentials and 32-bit sums, and by what a
    probability loses below fp16's normal range."""
    n, Hq = 2000, 3
    g = torch.Generator().manual_seed(17)
    c = torch.tensor([1.0, 1.5, 2.0, 3.0, 4.0, 6.0])[torch.randint(0, 6, (n,), generator=g)]
    k = torch.zeros((n, 1, D))
    k[:, 0, 0] = c * (2.0 ** (power // 2) * sign)
    v = _normal((n, 1, D), 18) * torch.exp2(torch.randint(-8, 9, (n, 1, 1), generator=g).float())
    q = torch.zeros((1, 1, Hq, D))
    q[..., 0] = 2.0 ** (power - power // 2)
    pool = Pool([(k, v)], 128, 1, D, 1)
    c = pool.held[0][0][:, 0, 0] * sign                 # what 4 bits hold of them, eight bits each
    out = torch.empty((1, 1, Hq, D), dtype=torch.bfloat16, device=DEV)
    pool.call(hsa, q.to(torch.bfloat16).to(DEV), out, _ws(hsa, 1, 1, Hq, 1, D), 0.6931471805599453)
    assert hsa.hsa_get_device_error() == 0
    best = pool.held[0][1][(c * sign == (c * sign).max()), 0]
    want = best.mean(0)
    tol = 2.0 ** -8 * want.abs() + (ref.P_STEP + 2.0 ** -20) * best.abs().mean(0) + 2.0 ** -25 * best.abs().max()
    assert ((out[0, 0].double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_nan(hsa, D):
    """A key or a value row held as NaN reaches the rows that see it, every dimension, and no
    others: newest keys that some rows may not see, and one that all see."""
    new, Hq, Hkv = 4, 8, 2
    for n, at in ((100, 98), (130, 127), (128, 125), (3, 1)):
        for which in (0, 1):
            kv = _random([n], Hkv, D, 11)
            pool = Pool(kv, 16, Hkv, D, 3)
            pool.words[which][int(pool.table[0, at // 16]), at % 16, 1] = -(1 << 24)    # s = 255
            q = _normal((1, new, Hq, D), 12).to(torch.bfloat16)
            out = torch.empty((1, new, Hq, D), dtype=torch.bfloat16, device=DEV)
            pool.call(hsa, q.to(DEV), out, _ws(hsa, 1, new, Hq, Hkv, D))
            got = out[0].double().cpu()
            want, tol = pool.want(0, q[0], new)
            clean = torch.ones((new, Hq), dtype=torch.bool)
            clean[max(0, at - (n - new)):, Hq // 2:] = False
            assert ((got - want).abs()[clean] <= tol[clean]).all()
            assert got[~clean].isnan().all()
    assert hsa.hsa_get_device_error() == 0


def test_bad_pages_and_lengths_are_reported(hsa):
    D, Hq, Hkv = 64, 4, 2
    pool = Pool(_random([40, 20], Hkv, D, 13), 16, Hkv, D, 13)
    q = _normal((2, 1, Hq, D), 1).to(torch.bfloat16)
    ws = _ws(hsa, 2, 1, Hq, Hkv, D)
    out = torch.empty((2, 1, Hq, D), dtype=torch.bfloat16, device=DEV)
    good = pool.table.clone()
    for bad in (-1, pool.codes[0].shape[0], 2 ** 31 - 1):
        pool.table = good.clone()
        pool.table[0, 1] = bad
        pool.call(hsa, q.to(DEV), out, ws)
        assert hsa.hsa_get_device_error() == -6
        k, v = (t.clone() for t in pool.held[0])        # the page reads as rows of zeros
        k[16:32], v[16:32] = 0.0, 0.0
        want, tol = base.attention(q[0].double(), k, v, [40], p_step=ref.P_STEP)
        assert ((out[0].double().cpu() - want).abs() <= tol + 1e-6).all()
    pool.table = good
    pool.lens = [-5, 20]
    pool.call(hsa, q.to(DEV), out, ws)
    assert hsa.hsa_get_device_error() == -6 and (out[0] == 0).all()
    pool.table = good[:, :2].contiguous()
    pool.lens = [40, 20]
    pool.call(hsa, q.to(DEV), out, ws)
    assert hsa.hsa_get_device_error() == -6
    want, tol = base.attention(q[0].double(), pool.held[0][0][:32], pool.held[0][1][:32], [32], p_step=ref.P_STEP)
    assert ((out[0].double().cpu() - want).abs() <= tol + 1e-6).all()


def test_same_result_in_any_company(hsa):
    """A call's result has the same bits alone and beside another stream's calls, each with a
    workspace of its own."""
    pool = Pool(_random([5000, 77], 2, 128, 16), 32, 2, 128, 16)
    q = _normal((2, 1, 8, 128), 1).to(torch.bfloat16).to(DEV)
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


def test_pages_past_4_gib(hsa):
    page, Hkv, Hq, D, n = 64, 8, 16, 128, 130
    P = (1 << 32) // (page * Hkv * D // 2) + 10
    kp, vp = (torch.empty((P, page, Hkv, D // 2), dtype=torch.uint8, device=DEV) for _ in "kv")
    words = [torch.empty((P, page, Hkv), dtype=torch.int32, device=DEV) for _ in "kv"]
    x = [_normal((n, Hkv, D), s).to(torch.bfloat16) for s in (3, 4)]
    table = torch.tensor([[P - 1, P - 3, P - 2]], dtype=torch.int32, device=DEV)
    at = torch.arange(n)
    slots = (table[0].cpu().long()[at // page] * page + at % page).int().to(DEV)
    hsa.hsa_kv4_quant_scatter(kp, vp, *words, *(t.to(DEV) for t in x), slots, n)
    held = [_held(t) for t in x]
    q = _normal((1, 1, Hq, D), 5).to(torch.bfloat16)
    out = torch.empty((1, 1, Hq, D), dtype=torch.bfloat16, device=DEV)
    hsa.hsa_paged_attention(q.to(DEV), kp, vp, table, torch.tensor([n], dtype=torch.int32, device=DEV), out,
                            k_scale=words[0], v_scale=words[1], workspace=_ws(hsa, 1, 1, Hq, Hkv, D))
    assert hsa.hsa_get_device_error() == 0
    want, tol = base.attention(q[0].double(), held[0][2], held[1][2], [n], p_step=ref.P_STEP)
    tol = tol + ref.small_weights(q[0].double(), held[0][2], held[1][1], [n])
    assert ((out[0].double().cpu() - want).abs() <= tol).all()


FAR = [(30, 119), (30, 126), (60, 118), (60, 126), (-30, 126), (-60, -62), (-60, -90), (30, -95), (60, -95), (-60, 119)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("level,power", FAR)
@pytest.mark.parametrize("n,new", [(100, 1), (7000, 1), (300, 3)])
def test_scores_away_from_zero_beside_values_at_the_ends(hsa, n, new, level, power, D):
    """All scores near 2^level's exponent, values near 2^power: the result is a mean of values,
    whatever the two add up to; in one block and joined."""
    g = torch.Generator().manual_seed(n + power)
    k = torch.zeros((n, 1, D))
    k[:, 0, 0] = level + 3 * torch.rand((n,), generator=g) - 1.5
    q = torch.zeros((1, new, 2, D))
    q[..., 0] = 1.0
    v = (torch.rand((n, 1, D), generator=g) + 0.9) * 2.0 ** power
    _compare(hsa, [(k, v)], q.to(torch.bfloat16), 128, scale=0.6931471805599453)
