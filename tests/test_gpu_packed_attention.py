"""Attention over packed sequences against the 64-bit reference: masks, groups, lengths from
none on, continued prompts, strided rows, what lies behind the sequences, NaN in places that
a row does not see, splitting along the keys, and the use together with the paged cache."""
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


def _cum(ns, first=0):
    out = [first]
    for n in ns:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32)


def _data(lens, Hq, Hkv, D, seed, lead=0, trail=0, size=1.0):
    """q, k, v with NaN in the rows before and behind the sequences."""
    g = torch.Generator().manual_seed(seed)
    tq, tk = sum(a for a, _ in lens), sum(b for _, b in lens)
    out = []
    for n, H in ((tq, Hq), (tk, Hkv), (tk, Hkv)):
        x = torch.full((lead + n + trail, H, D), float("nan"))
        x[lead:lead + n] = torch.randn((n, H, D), generator=g)
        out.append(x.to(torch.bfloat16))
    out[0][lead:lead + tq] *= size
    return out, _cum([a for a, _ in lens], lead), _cum([b for _, b in lens], lead)


def _compare(got, q, k, v, cu_q, cu_k, lens, mask, scale=None, rows=None):
    """rows: a step through the queries (the reference is slow)."""
    for b, (lq, lk) in enumerate(lens):
        at = range(0, lq, rows or 1)
        if lq and rows:
            at = sorted({*at, lq - 1})
        at = list(at)
        qs = q[int(cu_q[b]):int(cu_q[b]) + lq][at].double()
        ks, vs = (t[int(cu_k[b]):int(cu_k[b]) + lk].double() for t in (k, v))
        want, tol = ref.attention(qs, ks, vs, ref.limits(lq, lk, mask)[at], scale)
        err = (got[int(cu_q[b]):int(cu_q[b]) + lq][at].double() - want).abs()
        assert (err <= tol).all(), (b, lq, lk, float((err / tol).nan_to_num(9e9).max()))


def _check(hsa, lens, Hq, Hkv, D, mask, seed, lead=0, trail=0, split=True, rows=None, size=1.0, scale=0.0):
    (q, k, v), cu_q, cu_k = _data(lens, Hq, Hkv, D, seed, lead, trail, size)
    out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(hsa.hsa_packed_attention_workspace_bytes(Hq, Hkv, D), dtype=torch.uint8,
                     device=DEV) if split else None
    hsa.hsa_packed_attention(q.to(DEV), k.to(DEV), v.to(DEV), cu_q.to(DEV), cu_k.to(DEV), out, mask=mask,
                             scale=scale, workspace=ws)
    assert hsa.hsa_get_device_error() == 0
    got = out.cpu()
    assert (got[:lead] == 9.0).all() and (got[int(cu_q[-1]):] == 9.0).all()
    _compare(got, q, k, v, cu_q, cu_k, lens, mask, scale or None, rows)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [0, 1, 7])
@pytest.mark.parametrize("n", [1, 2, 127, 128, 129, 300])
def test_one_sequence(hsa, n, mask, D):
    _check(hsa, [(n, n)], 2, 1, D, mask, n + mask)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (6, 2), (5, 1), (16, 2), (40, 1)])
def test_groups(hsa, Hq, Hkv, D):
    _check(hsa, [(70, 70), (33, 33)], Hq, Hkv, D, 1, Hq)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [0, 1, 50])
def test_ragged_sequences_between_rows_of_nan(hsa, mask, D):
    """Lengths of none and one among others; the rows before and behind the sequences hold
    NaN and keep their outputs."""
    lens = [(5, 5), (0, 0), (200, 200), (1, 1), (0, 40), (129, 129), (64, 64)]
    _check(hsa, lens, 4, 2, D, mask, 3, lead=3, trail=130)
    _check(hsa, lens, 4, 2, D, mask, 4, lead=3, trail=130, split=False)


@pytest.mark.parametrize("mask", [0, 1, 16])
def test_more_queries_than_keys(hsa, mask):
    """The first queries of a masked sequence then see nothing, and a sequence without keys
    is zeros; some units have no key at all."""
    _check(hsa, [(300, 40), (10, 0), (400, 3)], 2, 2, 64, mask, 5)
    _check(hsa, [(600, 129)], 2, 1, 128, mask, 6)
    _check(hsa, [(10, 0)], 2, 1, 128, mask, 7)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [0, 1, 100])
def test_continued_prompts_are_split_along_the_keys(hsa, mask, D):
    """Few units with long keys: cut into pieces and joined; without a workspace, whole."""
    lens = [(3, 2500), (70, 5000), (1, 700), (5, 100)]
    _check(hsa, lens, 4, 1, D, mask, 8, rows=9)
    _check(hsa, lens, 4, 1, D, mask, 8, rows=9, split=False)


@pytest.mark.parametrize("mask", [0, 1])
def test_more_units_than_a_wave(hsa, mask):
    """More units than SMs: whole waves, and without a mask a cut last wave."""
    _check(hsa, [(1100, 1100), (515, 515)], 32, 8, 128, mask, 9, rows=131)
    _check(hsa, [(900, 900)], 48, 48, 64, mask, 10, rows=131)


def test_many_sequences(hsa):
    """More sequences than lanes of a warp."""
    lens = [((7 * b) % 40, (7 * b) % 40 + b % 3) for b in range(150)]
    _check(hsa, lens, 2, 1, 64, 1, 11)


@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_hundreds(hsa, D):
    """Large scores, so that the running maximum moves late and O is rescaled."""
    _check(hsa, [(700, 700)], 2, 1, D, 1, 12, size=12.0)
    _check(hsa, [(300, 900)], 2, 1, D, 0, 13, size=12.0)
    _check(hsa, [(100, 100)], 2, 1, D, 1, 14, scale=0.5)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_a_fused_projection(hsa, D):
    """q, k and v as slices of one [tokens, (Hq + 2 Hkv) D] tensor."""
    Hq, Hkv, n = 6, 2, 333
    x = torch.randn((n, (Hq + 2 * Hkv) * D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    xd = x.to(DEV)

    def parts(t):
        return [y.unflatten(1, (-1, D)) for y in t.split([Hq * D, Hkv * D, Hkv * D], 1)]
    cu = _cum([100, 233])
    out = torch.empty((n, Hq, D), dtype=torch.bfloat16, device=DEV)
    hsa.hsa_packed_attention(*parts(xd), cu.to(DEV), cu.to(DEV), out, mask=1)
    assert hsa.hsa_get_device_error() == 0
    _compare(out.cpu(), *parts(x), cu, cu, [(100, 100), (233, 233)], 1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("split", [False, True])
def test_nan_and_infinity_reach_only_rows_that_see_them(hsa, D, split):
    """K and V of some tokens hold NaN or infinity: rows that do not see those tokens have
    their usual results, in their own sequence and in the others."""
    for mask, lens in ((1, [(200, 200), (150, 150)]), (60, [(200, 200), (150, 150)]), (1, [(40, 1700)])):
        Hq, Hkv = 4, 2
        (q, k, v), cu_q, cu_k = _data(lens, Hq, Hkv, D, 15)
        lq, lk = lens[0]
        spoiled = [(lk - 25, 0, float("nan")), (lk - 3, 1, float("inf"))]
        v0, k0 = v.clone(), k.clone()
        for at, h, x in spoiled:
            v[at, h, 5] = x
            k[at, h, 9] = float("nan")
        v[lk - 1, 0, :] = float("-inf")
        out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(hsa.hsa_packed_attention_workspace_bytes(Hq, Hkv, D), dtype=torch.uint8,
                         device=DEV) if split else None
        hsa.hsa_packed_attention(q.to(DEV), k.to(DEV), v.to(DEV), cu_q.to(DEV), cu_k.to(DEV), out, mask=mask,
                                 workspace=ws)
        assert hsa.hsa_get_device_error() == 0
        got = out.cpu()
        limit = torch.from_numpy(ref.limits(lq, lk, mask))
        want, tol = ref.attention(q[:lq].double(), k0[:lk].double(), v0[:lk].double(), limit)
        for h in range(Hq):
            first = min(at for at, hk, _ in spoiled + [(lk - 1, 0, 0)] if hk == h // (Hq // Hkv))
            blind = limit <= first
            err = (got[:lq, h].double() - want[:, h]).abs()[blind]
            assert (err <= tol[:, h][blind]).all()
            assert got[:lq, h][~blind].isnan().any(-1).all()
        _compare(got[lq:], q[lq:], k0[lk:], v0[lk:], cu_q[1:] - lq, cu_k[1:] - lk, lens[1:], mask)


def test_offsets_out_of_range_are_reported(hsa):
    (q, k, v), cu_q, cu_k = _data([(50, 50), (60, 60)], 2, 1, 64, 16)
    q, k, v = q.to(DEV), k.to(DEV), v.to(DEV)
    for bad_q, bad_k in (([0, 50, 111], [0, 50, 110]), ([0, 50, 110], [0, 50, 2 ** 31 - 1]),
                         ([-4, 50, 110], [0, 50, 110]), ([0, 80, 50], [0, 50, 110]),
                         ([0, 50, 110], [0, 110, 50]), ([0, 2 ** 31 - 1, -2 ** 31], [5, -1, 7])):
        guard = torch.full((140, 2, 64), 9.0, dtype=torch.bfloat16, device=DEV)
        out = guard[:110]
        hsa.hsa_packed_attention(q, k, v, torch.tensor(bad_q, dtype=torch.int32, device=DEV),
                                 torch.tensor(bad_k, dtype=torch.int32, device=DEV), out, mask=1)
        assert hsa.hsa_get_device_error() == -6
        assert (guard[110:] == 9.0).all()
    # and the device is as it was
    _check(hsa, [(50, 50), (60, 60)], 2, 1, 64, 1, 16)


def test_captured_call_follows_the_offsets(hsa):
    """One captured call serves batches of other lengths within the same buffers."""
    Hq, Hkv, D, cap = 4, 2, 64, 900
    q, k, v = (torch.empty((cap, H, D), dtype=torch.bfloat16, device=DEV) for H in (Hq, Hkv, Hkv))
    cu_q, cu_k = (torch.zeros(4, dtype=torch.int32, device=DEV) for _ in range(2))
    out = torch.empty_like(q)
    ws = torch.empty(hsa.hsa_packed_attention_workspace_bytes(Hq, Hkv, D), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            hsa.hsa_packed_attention(q, k, v, cu_q, cu_k, out, mask=1, workspace=ws)
        for i, lens in enumerate(([(10, 10), (300, 300), (0, 0)], [(400, 400), (5, 400), (90, 90)],
                                  [(0, 0), (0, 0), (1, 1)])):
            data, cq, ck = _data(lens, Hq, Hkv, D, 20 + i)
            for t, x in zip((q, k, v), data):
                t.fill_(float("nan"))
                t[:x.shape[0]] = x
            cu_q.copy_(cq)
            cu_k.copy_(ck)
            out.fill_(9.0)
            graph.replay()
            side.synchronize()
            _compare(out.cpu(), *data, cq, ck, lens, 1)
            assert (out[int(cq[-1]):] == 9.0).all()
    assert hsa.hsa_get_device_error() == 0


def test_same_bits_beside_another_stream(hsa):
    (q, k, v), cu_q, cu_k = _data([(300, 3000), (40, 900)], 8, 2, 128, 17)
    q, k, v, cu_q, cu_k = (t.to(DEV) for t in (q, k, v, cu_q, cu_k))
    size = hsa.hsa_packed_attention_workspace_bytes(8, 2, 128)
    outs = [torch.empty_like(q) for _ in range(3)]
    wss = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(2)]
    hsa.hsa_packed_attention(q, k, v, cu_q, cu_k, outs[0], mask=1, workspace=wss[0])
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(torch.cuda.Stream()):
            hsa.hsa_packed_attention(q, k, v, cu_q, cu_k, outs[1 + i], mask=1, workspace=wss[i])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("D", [64, 128])
def test_wait_timeout_is_reported(hsa, D):
    """A withheld signal (no fault): the bounded wait runs out, the call reports it and the
    device goes on."""
    (q, k, v), cu_q, cu_k = _data([(300, 300)], 2, 1, D, 18)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    hsa.hsa_test_inject_attention_stall(1)
    try:
        hsa.hsa_packed_attention(q.to(DEV), k.to(DEV), v.to(DEV), cu_q.to(DEV), cu_k.to(DEV), out, mask=1)
        assert hsa.hsa_get_device_error() == -7
    finally:
        hsa.hsa_test_inject_attention_stall(0)
    _check(hsa, [(300, 300)], 2, 1, D, 1, 18)


@pytest.mark.parametrize("f8", [False, True])
def test_prompts_then_tokens(hsa, f8):
    """Serving: prompts in one packed call, their K/V into the paged cache (bf16 or 8-bit),
    then tokens one by one from the pages.  The tokens' results equal those of the reference
    over the values that the cache holds."""
    Hq, Hkv, D, page, steps = 8, 2, 64, 16, 3
    lens = [37, 5, 64]
    B, P = len(lens), 16
    (q, k, v), cu, _ = _data([(n, n) for n in lens], Hq, Hkv, D, 19)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    kd, vd = k.to(DEV), v.to(DEV)
    hsa.hsa_packed_attention(q.to(DEV), kd, vd, cu.to(DEV), cu.to(DEV), out, mask=1)
    _compare(out.cpu(), q, k, v, cu, cu, [(n, n) for n in lens], 1)
    order = torch.randperm(P, generator=torch.Generator().manual_seed(2)).int()
    table = order[:B * 5].view(B, 5) if B * 5 <= P else None
    slots = torch.cat([table[b, torch.arange(n) // page] * page + torch.arange(n) % page
                       for b, n in enumerate(lens)]).int()
    shape = (P, page, Hkv, D)
    if f8:
        kp, vp = (torch.zeros(shape, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
        ks, vs = (torch.zeros(shape[:3], dtype=torch.uint8, device=DEV) for _ in range(2))

        def write(x, y, at):
            hsa.hsa_kv_quant_scatter(kp, vp, ks, vs, x, y, at, at.numel())
    else:
        kp, vp = (torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ks = vs = None

        def write(x, y, at):
            hsa.hsa_kv_sync_scatter(kp.view(-1, Hkv, D), vp.view(-1, Hkv, D), x, y, at, at.numel())
    write(kd, vd, slots.to(DEV))

    def held(x):
        return torch.from_numpy(ref.values(*ref.quantise_rows(x.double().numpy())[:2])) if f8 else x.double()
    cache = [[held(t[int(cu[b]):int(cu[b + 1])]) for t in (k, v)] for b in range(B)]
    ws = torch.empty(hsa.hsa_paged_attention_workspace_bytes(B, 1, Hq, Hkv, D), dtype=torch.uint8, device=DEV)
    g = torch.Generator().manual_seed(3)
    for step in range(steps):
        x, y = (torch.randn((B, Hkv, D), generator=g).to(torch.bfloat16) for _ in range(2))
        qn = torch.randn((B, 1, Hq, D), generator=g).to(torch.bfloat16)
        at = torch.tensor([int(table[b, (n + step) // page]) * page + (n + step) % page
                           for b, n in enumerate(lens)], dtype=torch.int32)
        write(x.to(DEV), y.to(DEV), at.to(DEV))
        now = torch.tensor([n + step + 1 for n in lens], dtype=torch.int32)
        one = torch.empty((B, 1, Hq, D), dtype=torch.bfloat16, device=DEV)
        hsa.hsa_paged_attention(qn.to(DEV), kp, vp, table.contiguous().to(DEV), now.to(DEV), one, k_scale=ks,
                                v_scale=vs, workspace=ws)
        for b in range(B):
            cache[b] = [torch.cat([c, held(t[b:b + 1])]) for c, t in zip(cache[b], (x, y))]
            want, tol = ref.attention(qn[b].double(), *cache[b], [int(now[b])],
                                      p_step=2.0 ** -11 if f8 else 2.0 ** -8)
            assert ((one[b].double().cpu() - want).abs() <= tol).all()
    assert hsa.hsa_get_device_error() == 0


def test_rows_of_one_head_in_a_wider_tensor(hsa):
    """One head's rows as a slice whose head dimension has any stride."""
    x = torch.randn((50, 3 * 64), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    xd = x.to(DEV)

    def part(t, i):
        return t.as_strided((50, 1, 64), (192, 7, 1), 64 * i)
    cu = _cum([50])
    out = torch.empty((50, 1, 64), dtype=torch.bfloat16, device=DEV)
    hsa.hsa_packed_attention(*(part(xd, i) for i in range(3)), cu.to(DEV), cu.to(DEV), out, mask=1)
    _compare(out.cpu(), *(part(x, i) for i in range(3)), cu, cu, [(50, 50)], 1)


# ---------- many more blocks than SMs: a block takes several units, in an order that may differ

def _mixed(seed, batch=52):
    """Sequences of none to 300 queries: continued, plain, without keys, or of fewer keys than
    queries (whose first rows see nothing under a mask)."""
    g = torch.Generator().manual_seed(seed)
    lens = []
    for b in range(batch):
        n = int(torch.randint(0, 60, (), generator=g)) + (250 if b % 13 == 5 else 0)
        lens.append((n, (n, n + 200, 0, n // 3, n + 1)[b % 5]))
    return lens


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [0, 1, 24])
@pytest.mark.parametrize("G", [1, 3, 4, 64])
def test_blocks_take_several_units(hsa, G, mask, D):
    """The query rows come by TMA or (G = 3) by the warps, the output rows go by TMA in boxes
    of 32 or (G = 3, 64, and the last rows) by the warps."""
    _check(hsa, _mixed(30 + G), 8 * G, 8, D, mask, 31, lead=2, trail=40,
           rows=11 if G < 64 else 200)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mask", [0, 1])
def test_same_bits_whichever_block_takes_a_unit(hsa, mask, D):
    lens = [(90 + 11 * (b % 7), 90 + 300 * (b % 3)) for b in range(60)]
    (q, k, v), cu_q, cu_k = _data(lens, 8, 4, D, 32)
    q, k, v, cu_q, cu_k = (t.to(DEV) for t in (q, k, v, cu_q, cu_k))
    ws = torch.empty(hsa.hsa_packed_attention_workspace_bytes(8, 4, D), dtype=torch.uint8,
                     device=DEV)
    outs = [torch.full_like(q, 9.0) for _ in range(6)]
    for out in outs:
        hsa.hsa_packed_attention(q, k, v, cu_q, cu_k, out, mask=mask, workspace=ws)
    assert hsa.hsa_get_device_error() == 0
    assert all(torch.equal(outs[0], out) for out in outs[1:])
    _compare(outs[0].cpu(), q.cpu(), k.cpu(), v.cpu(), cu_q, cu_k, lens, mask, rows=67)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [2, 3])
def test_nan_between_units_of_a_block(hsa, G, D):
    """The last key of every third sequence holds NaN and infinity: rows that do not see it,
    and the other sequences', have their usual results."""
    Hkv, lens = 8, [(40 + 7 * (b % 5), 40 + 7 * (b % 5) + 130 * (b % 2)) for b in range(45)]
    (q, k, v), cu_q, cu_k = _data(lens, G * Hkv, Hkv, D, 33)
    v0, k0 = v.clone(), k.clone()
    for b in range(0, 45, 3):
        at = int(cu_k[b + 1]) - 1
        v[at, :, 3], v[at, :, D - 1] = float("nan"), float("-inf")
        k[at, :, 7] = float("inf")
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    hsa.hsa_packed_attention(*(t.to(DEV) for t in (q, k, v, cu_q, cu_k)), out, mask=1)
    assert hsa.hsa_get_device_error() == 0
    got = out.cpu()
    for b in range(0, 45, 3):
        last = int(cu_q[b + 1]) - 1
        assert got[last].isnan().any(-1).all()
        one = (torch.tensor([0]), torch.tensor([0]))
        lq, lk = lens[b]
        first, key = int(cu_q[b]), int(cu_k[b])
        # all rows but the last see none of it: a continued prompt one key shorter
        _compare(got[first:], q[first:], k0[key:], v0[key:], *one, [(lq - 1, lk - 1)], 1, rows=7)
    others = [b for b in range(45) if b % 3]
    for b in others:
        _compare(got[int(cu_q[b]):], q[int(cu_q[b]):], k0[int(cu_k[b]):], v0[int(cu_k[b]):],
                 torch.tensor([0]), torch.tensor([0]), [lens[b]], 1, rows=13)


def test_many_bad_offsets(hsa):
    """Offsets that fall and overlap make more rows than there are: reported, and nothing is
    written behind the output."""
    n, batch = 700, 300
    q, k, v = (torch.randn((n, H, 64), device=DEV).to(torch.bfloat16) for H in (4, 2, 2))
    ws = torch.empty(hsa.hsa_packed_attention_workspace_bytes(4, 2, 64), dtype=torch.uint8,
                     device=DEV)
    guard = torch.full((n + 300, 4, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    bad = torch.tensor([n * (b % 2) for b in range(batch + 1)], dtype=torch.int32, device=DEV)
    rising = torch.arange(batch + 1, dtype=torch.int32, device=DEV)
    for cu_q, cu_k in ((bad, bad), (bad, rising), (rising, bad)):
        for w in (None, ws):
            hsa.hsa_packed_attention(q, k, v, cu_q, cu_k, guard[:n], mask=1, workspace=w)
            assert hsa.hsa_get_device_error() == -6
            assert (guard[n:] == 9.0).all()
    _check(hsa, _mixed(3), 8, 4, 64, 1, 34, rows=7)


def test_captured_call_of_many_blocks_follows_the_offsets(hsa):
    """The grid is that of the buffers; the units of a replay are those of its offsets, from
    none to more than there are SMs."""
    Hq, Hkv, D, cap, batch = 16, 8, 128, 2200, 48
    q, k, v = (torch.empty((cap, H, D), dtype=torch.bfloat16, device=DEV) for H in (Hq, Hkv, Hkv))
    cu_q, cu_k = (torch.zeros(batch + 1, dtype=torch.int32, device=DEV) for _ in range(2))
    out = torch.empty_like(q)
    ws = torch.empty(hsa.hsa_packed_attention_workspace_bytes(Hq, Hkv, D), dtype=torch.uint8,
                     device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            hsa.hsa_packed_attention(q, k, v, cu_q, cu_k, out, mask=1, workspace=ws)
        for i, lens in enumerate(([(45, 45)] * batch, [(0, 0)] * batch,
                                  [(0, 0)] * 20 + [(30, 2100)] + [(0, 0)] * 27,
                                  [(b, b) for b in range(batch)])):
            data, cq, ck = _data(lens, Hq, Hkv, D, 40 + i)
            for t, x in zip((q, k, v), data):
                t.fill_(float("nan"))
                t[:x.shape[0]] = x
            cu_q.copy_(cq)
            cu_k.copy_(ck)
            out.fill_(9.0)
            graph.replay()
            side.synchronize()
            _compare(out.cpu(), *data, cq, ck, lens, 1, rows=11)
            assert (out[int(cq[-1]):] == 9.0).all()
    assert hsa.hsa_get_device_error() == 0


@pytest.mark.parametrize("D", [64, 128])
def test_wait_timeout_where_blocks_take_several_units(hsa, D):
    """As test_wait_timeout_is_reported: the blocks give up after their bounded wait and take
    no further unit."""
    lens = [(40, 300)] * 45
    (q, k, v), cu_q, cu_k = _data(lens, 16, 8, D, 35)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    hsa.hsa_test_inject_attention_stall(1)
    try:
        hsa.hsa_packed_attention(*(t.to(DEV) for t in (q, k, v, cu_q, cu_k)), out, mask=1)
        assert hsa.hsa_get_device_error() == -7
    finally:
        hsa.hsa_test_inject_attention_stall(0)
    _check(hsa, lens, 16, 8, D, 1, 35, rows=13)


def test_rows_formed_again_over_long_keys(hsa):
    """Rows that took in a masked NaN are formed again on the CUDA cores, here for longer than
    the warps wait for one another, in blocks that have another unit to do."""
    H, D, lq, n, at = 8, 128, 10300, 1_200_000, 1_200_000 - 130
    g = torch.Generator(DEV).manual_seed(50)
    q, k, v = (torch.randn((m, H, D), generator=g, device=DEV, dtype=torch.bfloat16)
               for m in (lq, n, n))
    v[at] = float("nan")
    out = torch.full_like(q, 9.0)
    hsa.hsa_packed_attention(q, k, v, _cum([lq]).to(DEV), _cum([n]).to(DEV), out, mask=1)
    assert hsa.hsa_get_device_error() == 0
    first = lq - (n - at)   # the first row that sees the NaN
    nan = out.isnan()
    assert nan[first:].all() and not nan[:first].any()
    for h, row in ((0, first - 1), (7, first - 40), (3, 5000)):
        ks, vs = (t[:at, h:h + 1].cpu().double() for t in (k, v))
        want, tol = ref.attention(q[row:row + 1, h:h + 1].cpu().double(), ks, vs,
                                  [n - lq + row + 1])
        assert ((out[row, h].cpu().double() - want[0, 0]).abs() <= tol[0, 0]).all()


@pytest.mark.parametrize("mask", [0, 1])
def test_blocks_of_several_units_beside_another_stream(hsa, mask):
    """Two grids whose blocks take further units, at the same time: each takes its own."""
    lens = [(90 + 11 * (b % 7), 90 + 300 * (b % 3)) for b in range(60)]
    (q, k, v), cu_q, cu_k = _data(lens, 16, 8, 128, 36)
    q, k, v, cu_q, cu_k = (t.to(DEV) for t in (q, k, v, cu_q, cu_k))
    size = hsa.hsa_packed_attention_workspace_bytes(16, 8, 128)
    outs = [torch.full_like(q, 9.0) for _ in range(7)]
    wss = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(2)]
    hsa.hsa_packed_attention(q, k, v, cu_q, cu_k, outs[0], mask=mask, workspace=wss[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            hsa.hsa_packed_attention(q, k, v, cu_q, cu_k, outs[1 + i], mask=mask,
                                     workspace=wss[i % 2])
    torch.cuda.synchronize()
    assert hsa.hsa_get_device_error() == 0
    assert all(torch.equal(outs[0], out) for out in outs[1:])
