"""hsa_page_plan against the sequences taken one after another, number for number."""
import pytest
import torch

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


def _state(lens, page, cols, spare, seed, pages=None):
    """A table whose sequences hold distinct pages, and a stack of the others."""
    g = torch.Generator().manual_seed(seed)
    have = [-(-n // page) for n in lens]
    pages = sum(have) + spare if pages is None else pages
    ids = torch.randperm(pages, generator=g).int()
    table = torch.full((len(lens), cols), -5, dtype=torch.int32)
    at = 0
    for b, c in enumerate(have):
        table[b, :c] = ids[at:at + c]
        at += c
    free = torch.full((pages,), -7, dtype=torch.int32)
    free[:pages - at] = ids[at:]
    return table, free, pages - at


def _run(hsa, lens, want, page, table, free, n_free, max_new, max_keys, in_place=False):
    def dev(x):
        return torch.as_tensor(x, dtype=torch.int32).to(DEV).contiguous()
    B = len(lens)
    d = {"table": dev(table), "free": dev(free), "cu_q": dev([9] * (B + 1)), "cu_k": dev([9] * (B + 1)),
         "slots": dev([9] * max_new), "positions": dev([9] * max_new)}
    if max_keys is not None:
        d["key_rows"] = dev([9] * max_keys)
    ls, ws, nf = dev(lens), dev(want), dev([n_free])
    d["lens_out"] = ls if in_place else dev([9] * B)
    d["n_free_out"] = nf if in_place else dev([9])
    hsa.hsa_page_plan(ls, ws, page, d["table"], d["free"], nf, d["n_free_out"], d["lens_out"], d["cu_q"], d["slots"],
                      d["positions"], cu_k=d["cu_k"], key_rows=d.get("key_rows"))
    return d


def _check(hsa, lens, want, page, table, free, n_free, max_new, max_keys=None, in_place=False):
    got = _run(hsa, lens, want, page, table, free, n_free, max_new, max_keys, in_place)
    exp, bad = ref.plan(list(lens), list(want), page, table, free, n_free, max_new, max_keys)
    for k, v in exp.items():
        assert torch.equal(got[k].cpu(), v), k
    assert hsa.hsa_get_device_error() == (-6 if bad else 0)
    return exp


def _mix(B, page, seed, most):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, most, (B,), generator=g)
    grow = torch.randint(0, 3 * page, (B,), generator=g)
    kind = torch.randint(0, 5, (B,), generator=g)
    want = torch.where(kind == 0, torch.zeros_like(lens), lens + grow)      # ended
    want = torch.where(kind == 1, lens // 2, want)                          # withdrawn
    want = torch.where(kind == 2, lens + 1, want)                           # one token
    return lens.tolist(), want.tolist()


@pytest.mark.parametrize("B,page,most", [(1, 16, 40), (3, 1, 9), (64, 16, 300), (40, 64, 2000), (7, 256, 900),
                                         (1025, 8, 30), (2500, 4, 12)])
def test_mixed_steps(hsa, B, page, most):
    """Sequences that grow, end, are cut short and stand still; few and many rows to fill."""
    lens, want = _mix(B, page, B + page, most)
    cols = -(-(most + 3 * page) // page)
    table, free, n = _state(lens, page, cols, sum(3 for _ in lens) + 2, 5)
    new = sum(max(0, w - h) for h, w in zip(lens, want))
    keys = sum(want)
    for max_new, max_keys in ((new, keys), (new + 13, keys + 5), (new + 9000, None)):
        _check(hsa, lens, want, page, table, free, n, max_new, max_keys)
        _check(hsa, lens, want, page, table, free, n, max_new, max_keys, in_place=True)


@pytest.mark.parametrize("B", [1, 3, 200, 512, 513, 1024, 1025])
def test_decoders_steps(hsa, B):
    """A token each at most: sequences at every place in a page, some that stand still or end."""
    page = 8
    lens = [(5 * b) % 40 for b in range(B)]
    want = [0 if b % 7 == 3 else n if b % 11 == 5 else n + 1 for b, n in enumerate(lens)]
    table, free, n = _state(lens, page, 6, B // 3 + 1, 9)
    new = sum(w > h for h, w in zip(lens, want))
    for max_new in (new, new + 5, new // 2, new + 9000):
        for n_free in (n, n // 4, 0):
            _check(hsa, lens, want, page, table, free, n_free, max_new, in_place=n_free == n)
    _check(hsa, lens, want, page, table, free, n, new, sum(want))
    bad = table.clone()
    bad[B // 2, lens[B // 2] // page] = 1 << 20      # the page that a token goes to, or none
    _check(hsa, lens, want, page, bad, free, n, new)


@pytest.mark.parametrize("B", [6, 1300])
def test_pages_and_places_that_do_not_last(hsa, B):
    """What no longer grows keeps its length; what needs no page still does; nothing is reported."""
    page = 16
    lens = [(37 * b) % 50 for b in range(B)]
    want = [n + (5 if b % 3 else 40) for b, n in enumerate(lens)]
    asked = sum(w - h for h, w in zip(lens, want))
    need = sum(-(-w // page) - -(-h // page) for h, w in zip(lens, want))
    table, free, _ = _state(lens, page, 8, need, 3)
    for n_free in (0, 1, need // 2, need):
        for max_new in (0, 1, asked // 3, asked - 1, asked):
            exp = _check(hsa, lens, want, page, table, free, n_free, max_new)
            assert n_free < need or max_new < asked or exp["lens_out"].tolist() == want


def test_pages_go_round(hsa):
    """Step after step in place: no page is held twice, none is lost."""
    g = torch.Generator().manual_seed(3)
    B, page, cols, pages = 20, 8, 12, 130
    table, free, n = _state([0] * B, page, cols, 0, 1, pages)
    lens = [0] * B
    for step in range(40):
        want = [0 if torch.rand((), generator=g) < 0.1 else min(cols * page, x + int(torch.randint(0, 12, (), generator=g)))
                for x in lens]
        exp = _check(hsa, lens, want, page, table, free, n, 200, None, in_place=True)
        table, free, n, lens = exp["table"], exp["free"], int(exp["n_free_out"]), exp["lens_out"].tolist()
        held = [int(x) for b in range(B) for x in table[b, :-(-lens[b] // page)]]
        assert sorted(held + free[:n].tolist()) == list(range(pages))


def test_lengths_and_stacks_out_of_range(hsa):
    table, free, n = _state([20, 5, 33, 0], 16, 3, 8, 2)
    for lens, want in (([20, 5, 33, 0], [20, 49, 34, -1]), ([20, -3, 33, 0], [21, 1, 33, 2]),
                       ([20, 5, 33, 0], [0, 5, 1000, 1])):
        _check(hsa, lens, want, 16, table, free, n, 60, 200)
    lens, want = [20, 5, 33, 0], [25, 6, 40, 1]
    _check(hsa, lens, want, 16, table, free, -1, 60, 200)
    _check(hsa, lens, [0, 0, 0, 0], 16, table, free, free.numel() + 1, 60, 200)
    _check(hsa, lens, [0, 0, 0, 0], 16, table, free, free.numel() - 2, 60, 200)     # given back twice
    _check(hsa, lens, want, 16, table, free, n, 60, 70)                            # keys past the room
    # ids that are none: of a page that is given back, that is taken, and that holds tokens
    t = table.clone()
    t[2, 2] = 999
    _check(hsa, lens, [20, 5, 0, 0], 16, t, free, n, 60, 200)
    t[0, 1] = -1
    _check(hsa, lens, want, 16, t, free, n, 60, 200)
    f = free.clone()
    f[n - 1] = -7
    _check(hsa, lens, want, 16, table, f, n, 60, 200)


def test_no_sequences_and_no_room(hsa):
    table, free, n = _state([3], 4, 2, 3, 2)
    _check(hsa, [], [], 4, table[:0], free, n, 7, 5)
    _check(hsa, [], [], 4, table[:0], free, n, 0, None)
    _check(hsa, [3], [0], 4, table, free, n, 0, 0)
    _check(hsa, [3], [8], 4, table, free, n, 5, 9000)
    _check(hsa, [0], [0], 4, table[:, :0], free, n, 3, None)
    _check(hsa, [0], [0], 4, table, free[:0], 0, 3, None)


def test_far_lengths(hsa):
    """Lengths near 2^31 whose sums do not fit 32 bits."""
    page, cols = 1 << 20, 2047
    top = cols * page
    lens, want = [top - 3, top - page, 5, 0], [top, top - page + 2, 6, 4]
    table = torch.arange(cols, dtype=torch.int32).repeat(4, 1)    # shared pages
    free = torch.arange(cols - 1, -1, -1, dtype=torch.int32)
    _check(hsa, lens, want, page, table, free, 6, 12)
    _check(hsa, lens, want, page, table, free, 6, 5)
    _check(hsa, lens, [0, top, 0, top], page, table[:, :], free, 6, 2 ** 12)
    got = _run(hsa, [5, 2, top, top], [6, 3, top, top], page, table, free, 6, 2, 20)
    assert got["cu_k"].tolist() == [0, 6, 9, 9 + top, ref.MOST]
    assert got["key_rows"].tolist() == [0, 1, 2, 3, 4, 5, 0, 1, 2, 0] + list(range(1, 11))
    assert hsa.hsa_get_device_error() == -6


def test_launches_and_graph(hsa):
    lens, want = [10, 20, 30], [11, 0, 50]
    table, free, n = _state(lens, 8, 9, 20, 4)
    before = hsa.hsa_launch_count()
    _run(hsa, lens, want, 8, table, free, n, 30, None)
    assert hsa.hsa_launch_count() == before + 1
    _run(hsa, lens, want, 8, table, free, n, 30, 9000)
    assert hsa.hsa_launch_count() == before + 3

    def dev(x):
        return torch.as_tensor(x, dtype=torch.int32).to(DEV)
    d = [dev(x) for x in (lens, want, table, free, [n], [0] * 4, [0] * 30, [0] * 30)]
    ls, ws, tb, fr, nf, cq, sl, ps = d
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hsa.hsa_page_plan(ls, ws, 8, tb, fr, nf, nf, ls, cq, sl, ps)
    for step_want in ([12, 0, 51], [13, 9, 40], [12, 10, 41]):      # a decoder's steps, in place
        exp, bad = ref.plan(ls.tolist(), step_want, 8, tb.cpu(), fr.cpu(), int(nf), 30)
        ws.copy_(dev(step_want))
        graph.replay()
        torch.cuda.synchronize()
        for x, k in ((ls, "lens_out"), (tb, "table"), (fr, "free"), (nf, "n_free_out"), (cq, "cu_q"), (sl, "slots"),
                     (ps, "positions")):
            assert torch.equal(x.cpu(), exp[k]), k
    assert hsa.hsa_get_device_error() == 0


def test_pages_asked_for_count_across_groups_of_sequences(hsa):
    """A sequence that asks for more pages than there are stops those behind it that need any,
    wherever it stands."""
    for B in (5, 1024, 1025, 1026, 2049):
        lens, want = [0] * B, [48] + [0] * (B - 2) + [1]
        table, free, n = _state(lens, 16, 4, 9, 7)
        for n_free in range(5):
            exp = _check(hsa, lens, want, 16, table, free, n_free, 200)
            assert exp["lens_out"][-1] == (n_free == 4)
    lens, want = [0] * 1025, [2] + [0] * 1023 + [1]
    table, free, _ = _state(lens, 1, 4, 9, 7)
    exp = _check(hsa, lens, want, 1, table, free, 1, 200)
    assert not exp["lens_out"].any() and exp["n_free_out"].tolist() == [1]


@pytest.mark.parametrize("B", [1023, 1024, 1025, 1026, 1027, 1028, 1029, 1030, 2049])
def test_every_size_of_the_stack(hsa, B):
    """Mixed needs on both sides of a border of 1024 sequences; any number of free pages, and of
    places for tokens, from none to what is needed."""
    page = 4
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 9, (B,), generator=g)
    want = lens.clone()
    some = torch.cat([torch.arange(3), torch.randint(0, B, (25,), generator=g), torch.arange(B - 10, B)])
    want[some] += torch.randint(1, 4 * page, some.shape, generator=g)
    want[torch.randint(0, B, (4,), generator=g)] = 0
    lens, want = lens.tolist(), want.tolist()
    asked = sum(max(0, w - h) for h, w in zip(lens, want))
    need = sum(max(0, -(-w // page) - -(-h // page)) for h, w in zip(lens, want))
    table, free, n = _state(lens, page, 8, need, 3)
    for n_free in range(need + 1):
        _check(hsa, lens, want, page, table, free, n_free, asked)
    for max_new in range(0, asked + 1, 7):
        _check(hsa, lens, want, page, table, free, n, max_new)
        _check(hsa, lens, want, page, table, free, need // 2, max_new)
