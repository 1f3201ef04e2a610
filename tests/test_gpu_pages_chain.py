"""A server's steps with the page plan, the normed and rotated rows, the 4-bit cache and the
attention over it, one after another on one stream: prompts come in, are read back for the packed
attention, tokens follow, sequences end and their pages are taken by others.  Each call may start
beside the end of the one before; what they hand to one another is compared with the same calls
made one at a time, and with the whole computed in 64 bits."""
import pytest
import torch

import oracle
import reference_cache as base
import reference_pages as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32, BF = torch.int32, torch.bfloat16


@pytest.fixture(scope="module")
def hsa():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2605_06892_gb300 as m
    m.lib()
    torch.cuda.set_device(0)
    m.hsa_get_device_error()
    return m


class Server:
    B, page, pages, cols, room = 5, 16, 40, 12, 96

    def __init__(self, D, Hq, Hkv, across):
        self.D, self.Hq, self.Hkv, self.across = D, Hq, Hkv, across
        g = torch.Generator().manual_seed(5)

        def ints(*shape, fill=0):
            return torch.full(shape, fill, dtype=I32, device=DEV)
        self.table, self.cu_q, self.cu_k = ints(self.B, self.cols, fill=-9), ints(self.B + 1), ints(self.B + 1)
        self.free = torch.randperm(self.pages, generator=g).int().to(DEV)
        self.n_free, self.lens, self.want = ints(1, fill=self.pages), ints(self.B), ints(self.B)
        self.slots, self.at, self.rows = ints(self.room), ints(self.room), ints(600)
        self.codes = [torch.zeros((self.pages, self.page, Hkv, D // 2), dtype=torch.uint8, device=DEV) for _ in "kv"]
        self.words = [ints(self.pages, self.page, Hkv) for _ in "kv"]
        self.weights = [1 + 0.3 * torch.randn((H, D) if across else (D,), generator=g) for H in (Hq, Hkv)]
        self.angles = oracle.rope_table((1, 1, self.cols * self.page), D)
        self.dev = [t.to(DEV) for t in (*self.weights, self.angles)]
        self.qkv = torch.zeros((self.room, Hq + 2 * Hkv, D), dtype=BF, device=DEV)
        self.q, self.k = (torch.zeros((self.room, H, D), dtype=BF, device=DEV) for H in (Hq, Hkv))
        self.back = [torch.zeros((600, Hkv, D), dtype=BF, device=DEV) for _ in "kv"]
        self.out = torch.zeros((self.room, Hq, D), dtype=BF, device=DEV)
        self.token = torch.zeros((self.B, 1, Hq, D), dtype=BF, device=DEV)
        self.g = g

    def step(self, hsa, want, after=lambda: None, fresh=None):
        """All sequences to `want` tokens.  Returns copies of what the step made."""
        x = torch.randn(self.qkv.shape, generator=self.g).to(BF) if fresh is None else fresh
        self.want.copy_(torch.tensor(want, dtype=I32))
        self.qkv.copy_(x)
        q, k, v = self.qkv.split((self.Hq, self.Hkv, self.Hkv), 1)
        wq, wk, angles = self.dev
        ws = torch.empty(hsa.hsa_paged_attention_workspace_bytes(self.B, 1, self.Hq, self.Hkv, self.D),
                         dtype=torch.uint8, device=DEV)
        for call in (
            lambda: hsa.hsa_page_plan(self.lens, self.want, self.page, self.table, self.free, self.n_free, self.n_free,
                                      self.lens, self.cu_q, self.slots, self.at, cu_k=self.cu_k, key_rows=self.rows),
            lambda: hsa.hsa_qk_norm_rope(q, k, wq, wk, self.q, self.k, across=self.across, table=angles,
                                         table_idx=self.at),
            lambda: hsa.hsa_kv4_quant_scatter(*self.codes, *self.words, self.k, v, self.slots, self.room),
            lambda: hsa.hsa_kv4_dequant_gather(*self.codes, *self.words, self.rows, 600, *self.back),
            lambda: hsa.hsa_packed_attention(self.q, *self.back, self.cu_q, self.cu_k, self.out, mask=1),
            lambda: hsa.hsa_paged_attention(self.q[:self.B].view(self.B, 1, self.Hq, self.D), *self.codes, self.table,
                                            self.lens, self.token, k_scale=self.words[0], v_scale=self.words[1],
                                            workspace=ws),
        ):
            call()
            after()
        return [t.clone() for t in (self.lens, self.table, self.free, self.n_free, self.slots, self.at, self.rows,
                                    self.cu_q, self.cu_k, self.q, self.k, *self.codes, *self.words, *self.back,
                                    self.out, self.token)]


STEPS = ([20, 1, 0, 33, 7], [21, 2, 40, 34, 8], [22, 3, 41, 0, 9], [23, 4, 42, 17, 10], [0, 5, 43, 18, 90],
         [64, 6, 44, 19, 91], [65, 7, 45, 20, 92], [66, 40, 46, 21, 93])


@pytest.mark.parametrize("D,Hq,Hkv,across", [(64, 4, 2, False), (128, 8, 2, True)])
def test_steps_in_a_row_equal_steps_one_at_a_time(hsa, D, Hq, Hkv, across):
    def run(after):
        s, made = Server(D, Hq, Hkv, across), []
        for want in STEPS:
            made += s.step(hsa, want, after)
        torch.cuda.synchronize()
        return made
    alone = run(torch.cuda.synchronize)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(alone, run(lambda: None)))
    assert hsa.hsa_get_device_error() == 0


@pytest.mark.parametrize("D,Hq,Hkv,across", [(64, 4, 2, False), (128, 8, 2, True)])
def test_steps_against_64_bits(hsa, D, Hq, Hkv, across):
    """Every step's attention outputs against 64 bits over what the cache has been given: queries
    and keys as the normed call made them (its own tests hold them to 64 bits), K and V as 4 bits
    hold them, by the sequences' histories."""
    s = Server(D, Hq, Hkv, across)
    history = [[torch.zeros((0, Hkv, D), dtype=torch.float64) for _ in "kv"] for _ in range(s.B)]
    lens = [0] * s.B
    for want in STEPS:
        x = torch.randn(s.qkv.shape, generator=s.g).to(BF)
        made = [t.cpu() for t in s.step(hsa, want, fresh=x)]
        q, k, out, token = made[9].double(), made[10], made[17].double(), made[18].double()
        assert made[0].tolist() == want and hsa.hsa_get_device_error() == 0
        n = sum(max(0, w - h) for h, w in zip(lens, want))
        at = made[5][:n]
        for got, part, w in ((q[:n], x[:n, :Hq], s.weights[0]), (k[:n].double(), x[:n, Hq:Hq + Hkv], s.weights[1])):
            y, tol = ref.norm_rope(part, w, 1e-6, across, s.angles, at, 2.0 ** -8)
            assert ((got - y).abs() <= tol).all()
        i = 0
        for b in range(s.B):
            new = max(0, want[b] - lens[b])
            for j, y in enumerate((k[i:i + new], x[i:i + new, Hq + Hkv:])):
                held = torch.from_numpy(ref.quantise_rows(y.double().numpy())[0])
                history[b][j] = torch.cat([history[b][j], held])[:want[b]]
            if new:
                y, tol = base.attention(q[i:i + new], *history[b], base.limits(new, want[b], 1))
                assert ((out[i:i + new] - y).abs() <= tol).all()
            y, tol = base.attention(q[b:b + 1], *history[b], [want[b]], p_step=ref.P_STEP)
            assert ((token[b] - y).abs() <= tol + 1e-6).all()
            i += new
        lens = list(want)


def test_captured_step(hsa):
    """One captured step of a decoder, replayed with other wanted lengths and inputs, on a stream of
    its own, against the same steps made eagerly."""
    eager, s = Server(64, 4, 2, False), Server(64, 4, 2, False)
    for x in (eager, s):
        x.step(hsa, STEPS[0], fresh=torch.ones(s.qkv.shape, dtype=BF))
    q, k, v = s.qkv.split((4, 2, 2), 1)
    ws = torch.empty(hsa.hsa_paged_attention_workspace_bytes(5, 1, 4, 2, 64), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            hsa.hsa_page_plan(s.lens, s.want, 16, s.table, s.free, s.n_free, s.n_free, s.lens, s.cu_q, s.slots, s.at,
                              cu_k=s.cu_k, key_rows=s.rows)
            hsa.hsa_qk_norm_rope(q, k, *s.dev[:2], s.q, s.k, table=s.dev[2], table_idx=s.at)
            hsa.hsa_kv4_quant_scatter(*s.codes, *s.words, s.k, v, s.slots, s.room)
            hsa.hsa_kv4_dequant_gather(*s.codes, *s.words, s.rows, 600, *s.back)
            hsa.hsa_packed_attention(s.q, *s.back, s.cu_q, s.cu_k, s.out, mask=1)
            hsa.hsa_paged_attention(s.q[:5].view(5, 1, 4, 64), *s.codes, s.table, s.lens, s.token, k_scale=s.words[0],
                                    v_scale=s.words[1], workspace=ws)
        for want in STEPS[1:]:
            x = torch.randn(s.qkv.shape, generator=s.g).to(BF)
            s.want.copy_(torch.tensor(want, dtype=I32))
            s.qkv.copy_(x)
            graph.replay()
            side.synchronize()
            made = [t.clone() for t in (s.lens, s.table, s.free, s.n_free, s.slots, s.at, s.rows, s.cu_q, s.cu_k, s.q,
                                        s.k, *s.codes, *s.words, *s.back, s.out, s.token)]
            assert all(torch.equal(a, b) for a, b in zip(made, eager.step(hsa, want, fresh=x)))
    assert hsa.hsa_get_device_error() == 0
