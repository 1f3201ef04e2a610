"""8-bit paged attention where the weights' sum has far to go: long stretches of zero rows,
scale bytes as fresh memory holds them, values at the top of the range; where keys and queries
differ far in size; and where scores are very large.  Against the 64-bit reference, within its
bounds."""
import numpy as np
import pytest
import torch

import reference_cache as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
PAGE = 128


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
    """Codes, scale bytes and the values that they stand for, of rows x [n, Hkv, D]."""
    c, s, _ = ref.quantise_rows(x.to(torch.bfloat16).double().numpy())
    return torch.from_numpy(c.astype(np.uint8)), torch.from_numpy(s), torch.from_numpy(ref.values(c, s))


class Sequence:
    """The keys of one sequence, row by row; `at` (page, place) of each in the pool."""

    def __init__(self, k, v, zero_scale=None):
        n, Hkv, D = k.shape
        P = -(-n // PAGE)
        self.codes = [torch.zeros((P * PAGE, Hkv, D), dtype=torch.uint8) for _ in range(2)]
        self.scales = [torch.full((P * PAGE, Hkv), 27, dtype=torch.uint8) for _ in range(2)]
        self.held = []
        for i, x in enumerate((k, v)):
            some = x.flatten(1).abs().amax(1) > 0
            c, s, y = _held(x[some])
            full = torch.zeros((n, Hkv, D), dtype=torch.float64)
            full[some] = y
            self.held.append(full)
            self.codes[i][:n][some], self.scales[i][:n][some] = c, s
            if zero_scale is not None:
                self.scales[i][:n][~some] = zero_scale
        self.n, self.P = n, P

    def pool(self):
        Hkv, D = self.codes[0].shape[1:]
        return ([c.view(self.P, PAGE, Hkv, D).to(DEV) for c in self.codes],
                [s.view(self.P, PAGE, Hkv).to(DEV) for s in self.scales])


def _attend(hsa, q, codes, scales, table, lens, scale=0.0):
    B, new, Hq, D = q.shape
    Hkv = codes[0].shape[2]
    out = torch.full_like(q, 9.0, device=DEV)
    ws = torch.empty(hsa.hsa_paged_attention_workspace_bytes(B, new, Hq, Hkv, D), dtype=torch.uint8, device=DEV)
    hsa.hsa_paged_attention(q.to(DEV), *codes, table.to(DEV), lens.to(DEV), out, k_scale=scales[0],
                            v_scale=scales[1], scale=scale, workspace=ws)
    assert hsa.hsa_get_device_error() == 0
    return out.double().cpu()


def _check(hsa, seq, q, scale=None):
    new, n = q.shape[1], seq.n
    codes, scales = seq.pool()
    got = _attend(hsa, q, codes, scales, torch.arange(seq.P, dtype=torch.int32)[None],
                  torch.tensor([n], dtype=torch.int32), scale or 0.0)
    want, tol = ref.attention(q[0].double(), *seq.held, ref.limits(new, n, 1), scale, p_step=2.0 ** -11)
    assert want.abs().amax() > 0
    err = (got[0] - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


def _normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("new,Hq", [(1, 4), (2, 12)])
@pytest.mark.parametrize("D,zeros", [(128, 140000), (64, 280000)])
def test_long_stretch_of_zero_rows(hsa, D, zeros, new, Hq):
    """More zero rows than a lane group of the join can count at 2^114 each, then 100 others
    (8 and 24 rows of queries: one column block and more)."""
    k, v = torch.zeros((zeros + 100, 1, D)), torch.zeros((zeros + 100, 1, D))
    k[zeros:], v[zeros:] = _normal((100, 1, D), 1), _normal((100, 1, D), 2)
    _check(hsa, Sequence(k, v), _normal((1, new, Hq, D), 3).to(torch.bfloat16))


@pytest.mark.parametrize("D", [64, 128])
def test_zero_rows_within_one_run(hsa, D):
    """A batch so large that a block's own run holds more than 16384 zero rows: the sequences
    share the page of zeros."""
    zeros, B, Hq = 140 * PAGE, 700, 2
    k, v = torch.zeros((PAGE + 100, 1, D)), torch.zeros((PAGE + 100, 1, D))
    k[PAGE:], v[PAGE:] = _normal((100, 1, D), 4), _normal((100, 1, D), 5)
    seq = Sequence(k, v)
    table = torch.zeros((B, 141), dtype=torch.int32)
    table[:, 140] = 1
    q = _normal((1, 1, Hq, D), 6).to(torch.bfloat16).expand(B, 1, Hq, D).contiguous()
    got = _attend(hsa, q, *seq.pool(), table, torch.full((B,), zeros + 100, dtype=torch.int32))
    full = [torch.cat([torch.zeros((zeros, 1, D), dtype=torch.float64), x[PAGE:]]) for x in seq.held]
    want, tol = ref.attention(q[0].double(), *full, [zeros + 100], p_step=2.0 ** -11)
    assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", ["first", "last", "spread"])
def test_zero_rows_with_scale_bytes_of_fresh_memory(hsa, at, D):
    """Rows that were never written, in a cache that was made with zeros: their scale bytes
    are zero and they stand for zeros."""
    n = 300
    some = {"first": torch.arange(n) >= 200, "last": torch.arange(n) < 100, "spread": torch.arange(n) % 3 == 0}[at]
    k, v = (_normal((n, 2, D), s) * some[:, None, None] for s in (7, 8))
    _check(hsa, Sequence(k, v, zero_scale=0), _normal((1, 2, 8, D), 9).to(torch.bfloat16))


@pytest.mark.parametrize("D", [64, 128])
def test_small_weights_count_at_the_top_of_the_range(hsa, D):
    """Values up to 2^127: 60000 keys whose weights are about 2^-20 of one key's weigh a few
    per cent together."""
    n = 60001
    k = torch.zeros((n, 1, D))
    k[1:, 0, 0], k[0, 0, 0] = -16.0, 4.0          # scores 4 and -16 in units of log2
    q = torch.zeros((1, 1, 2, D))
    q[..., 0] = 1.0
    v = (torch.rand((n, 1, D), generator=torch.Generator().manual_seed(10)) * 0.5 + 0.5) * 2.0 ** 127
    _check(hsa, Sequence(k, v), q.to(torch.bfloat16), scale=0.6931471805599453)


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
    _check(hsa, Sequence(k, v), q.to(torch.bfloat16), scale=0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ek,eq", [(110, -112), (120, -100), (-98, 112), (100, 20), (-90, -30)])
def test_keys_and_queries_of_very_different_size(hsa, ek, eq, D):
    """Scores of ordinary size from keys of 2^ek and queries of 2^eq."""
    n = 200
    k, v = _normal((n, 2, D), 11) * 2.0 ** ek, _normal((n, 2, D), 12)
    k[5], k[77] = 0.0, 0.0                        # scores of exactly zero
    q = (_normal((1, 2, 4, D), 13) * 2.0 ** eq).to(torch.bfloat16)
    _check(hsa, Sequence(k, v), q, scale=D ** -0.5 * 2.0 ** -(ek + eq))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", [10, 20, 25, 26, 31, 60, 100])
def test_scores_of_any_size(hsa, D, sign, power):
    """Scores are small numbers times 2^power, exactly, so that the keys that share the largest
    have all the weight, in equal parts, whatever their values' sizes: off by the rounding of
    probabilities and output and by 2^-20 for the exponentials (2^-22.5) and 32-bit sums."""
    n, Hq = 2000, 3
    g = torch.Generator().manual_seed(17)
    c = torch.randint(1, 8, (n,), generator=g)
    k = torch.zeros((n, 1, D))
    k[:, 0, 0] = c * (2.0 ** (power // 2) * sign)
    v = _normal((n, 1, D), 18) * torch.exp2(torch.randint(-8, 9, (n, 1, 1), generator=g).float())
    q = torch.zeros((1, 1, Hq, D))
    q[..., 0] = 2.0 ** (power - power // 2)
    seq = Sequence(k, v)
    codes, scales = seq.pool()
    got = _attend(hsa, q.to(torch.bfloat16), codes, scales, torch.arange(seq.P, dtype=torch.int32)[None],
                  torch.tensor([n], dtype=torch.int32), 0.6931471805599453)[0, 0]
    best = seq.held[1][(c * sign == (c * sign).max()), 0]
    want = best.mean(0)
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -20) * best.abs().mean(0)
    assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("f8", [True, False])
@pytest.mark.parametrize("power", [12, 30, 50, 90])
def test_largest_score_takes_all(hsa, f8, D, power):
    """Scores of any digits times 2^power.  The largest is further from the next than the sums'
    rounding, so that the output is its value: off by the output's rounding, and by 2^-20 for
    the exponential and the division."""
    n, Hq = 2000, 4
    k, v = _normal((n, 1, D), 19) * 2.0 ** (power // 2), _normal((n, 1, D), 20)
    q = (_normal((1, 1, Hq, D), 21) * 2.0 ** (power - power // 2)).to(torch.bfloat16)
    k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    seq = Sequence(k, v)
    codes, scales = seq.pool()
    held = seq.held
    if not f8:
        held = [k.double(), v.double()]
        codes = [torch.nn.functional.pad(x, (0, 0, 0, 0, 0, seq.P * PAGE - n)).view(seq.P, PAGE, 1, D).to(DEV)
                 for x in (k, v)]
        scales = [None, None]
    got = _attend(hsa, q, codes, scales, torch.arange(seq.P, dtype=torch.int32)[None],
                  torch.tensor([n], dtype=torch.int32))[0, 0]
    s = (q[0, 0].double() @ held[0][:, 0].T) * D ** -0.5
    top, at = s.topk(2, dim=1)
    apart = (q[0, 0].double().abs() @ held[0][:, 0].abs().T).amax(1) * D ** -0.5 * (D + 2) * 2.0 ** -23
    assert ((top[:, 0] - top[:, 1]) > apart + 40).all()
    want = held[1][at[:, 0], 0]
    assert ((got - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs() + 2.0 ** -39 * want.abs().amax()).all()
