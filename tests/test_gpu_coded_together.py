"""The operators of a serving loop over a cache of 8-bit codes one after the other: append with rotation, attention, rules on logits, the choice of a token -- against the oracle, in a captured graph
whose replays see new lengths, on streams of their own, for a prompt and then single tokens and a tree."""
import numpy as np
import pytest
import torch

from oracle import operators as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H, KVH, D, PAGE, BLOCK, V = 8, 2, 64, 32, 16, 777
U = 2.0 ** -24


def pkg():
    import paper_2401_15077_amd
    return paper_2401_15077_amd


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


class Loop:
    """Two sequences that grow by one token a step; everything a step reads that changes lies in device tensors."""

    def __init__(self, dtype, cache, seed, cap=128):
        p = pkg()
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.cap, pages = cap, 2 * cap // PAGE
        self.kc, self.vc = (torch.zeros(pages, KVH, PAGE, D, dtype=torch.int8, device=DEV).view(cache) for _ in range(2))
        self.ks, self.vs = (torch.zeros(pages, KVH, PAGE // BLOCK, device=DEV) for _ in range(2))
        self.table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32).view(2, -1).to(DEV)
        self.key_len = i32([3, 20])
        self.q, self.k, self.v = (torch.zeros(2, h, D, dtype=dtype, device=DEV) for h in (H, KVH, KVH))
        self.qr, self.out = torch.zeros_like(self.q), torch.zeros_like(self.q)
        self.logits, self.ruled, self.uniform = torch.zeros(2, V, device=DEV), torch.zeros(2, V, device=DEV), torch.zeros(2, device=DEV)
        self.text, self.n_text = torch.zeros(2, cap, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
        self.token, self.logprob = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV)
        self.chunk = p.Chunk(i32([0, 1, 2]), self.key_len, 2, 1, cap)
        self.kv = p.PagedKV8(self.kc, self.vc, self.table, self.ks, self.vs)
        self.plan = p.rope_plan(D, scaling="linear", factor=2.0)
        self.rules = p.LogitRules(self.text, self.n_text, repetition=torch.tensor([1.2, 1.5], device=DEV), frequency=torch.tensor([0.5, 0.25], device=DEV))
        self.filters = dict(temperature=torch.tensor([0.8, 1.2], device=DEV), top_k=i32([30, 0]), top_p=torch.tensor([0.9, 0.8], device=DEV), min_p=torch.tensor([0.0, 0.01], device=DEV))
        self.ws = torch.empty(p.chunk_attention_workspace(self.q, self.kv, self.chunk), dtype=torch.uint8, device=DEV)
        self.ws2 = torch.empty(p.sample_workspace(self.logits), dtype=torch.uint8, device=DEV)
        # the prompts, appended at once
        k, v = (torch.randn(23, KVH, D, device=DEV, generator=self.gen).to(dtype) for _ in range(2))
        p.rope(self.plan, None, k, v, chunk=p.Chunk(i32([0, 3, 23]), self.key_len, 23, 20, cap), kv=self.kv)

    def inputs(self, step):
        for t in (self.q, self.k, self.v, self.logits):
            t.copy_(torch.randn(t.shape, device=DEV, generator=self.gen) * (2.0 if t is self.logits else 1.0 + 0.2 * (step % 7)))
        self.uniform.copy_(torch.rand(2, device=DEV, generator=self.gen))
        self.key_len += 1

    def calls(self):
        p = pkg()
        p.rope(self.plan, self.q, self.k, self.v, chunk=self.chunk, kv=self.kv, q_out=self.qr)
        p.chunk_attention(self.qr, self.kv, self.chunk, window=30, softcap=8.0, out=self.out, workspace=self.ws)
        p.apply_logit_rules(self.logits, self.rules, out=self.ruled)
        p.sample(self.ruled, self.uniform, token=self.token, logprob=self.logprob, workspace=self.ws2, **self.filters)

    def results(self):
        return [t.clone() for t in (self.qr, self.out, self.ruled, self.token, self.logprob, self.ks, self.vs, self.kc.view(torch.uint8), self.vc.view(torch.uint8))]

    def after(self, step):                                        # the chosen token joins the text
        self.text[:, step] = self.token
        self.n_text.fill_(step + 1)

    def step(self, step):
        self.calls()
        r = self.results()
        self.after(step)
        return r


@pytest.mark.parametrize("cache", [torch.float8_e4m3fn, torch.int8], ids=str)
def test_a_loop_matches_the_oracle(cache):
    loop = Loop(torch.float32, cache, 1)
    e4m3 = cache == torch.float8_e4m3fn
    numbers = lambda c: ref.code_value(c.view(torch.uint8).cpu().numpy(), e4m3)
    f, table = ref.frequencies(D, scaling="linear", factor=2.0), loop.table.tolist()
    for step in range(40):                                        # past blocks, pages and the window
        loop.inputs(step)
        held = [(numbers(c), s.double().cpu().numpy()) for c, s in ((loop.kc, loop.ks), (loop.vc, loop.vs))]
        text = [loop.text[s, :step].tolist() for s in range(2)]
        loop.calls()
        keys = loop.key_len.tolist()
        rows = ref.chunk_rows([0, 1, 2], keys)
        pos = [r[3] for r in rows]
        turned, _ = ref.rotate(loop.k.double().cpu().numpy(), pos, f, D, False)
        kw = dict(page=PAGE, block=BLOCK, e4m3=e4m3, max_rows=1, max_keys=loop.cap, row_start=[0, 1, 2])
        for x, (values, scale), c, s in ((turned, held[0], loop.kc, loop.ks), (loop.v.double().cpu().numpy(), held[1], loop.vc, loop.vs)):
            want, want_scale, _ = ref.append_codes(x, values, scale, rows, table, keys, **kw)
            np.testing.assert_array_equal(s.double().cpu().numpy(), want_scale)
            np.testing.assert_array_equal(numbers(c), want)       # (no element of these lies within 2^-40 of a border)
        k, v = (numbers(c) * np.repeat(s.double().cpu().numpy(), BLOCK, axis=2)[..., None] for c, s in ((loop.kc, loop.ks), (loop.vc, loop.vs)))
        want, mean, big, count = ref.attention(loop.qr.double().cpu().numpy(), k, v, table, rows, 2, keys, page=PAGE, scale=D ** -0.5, softcap=8.0, window=30)
        tol = (2 * (64 * U * big + 5 * U * (big + 8.0)) + (count[:, None] / 8 + 33) * U)[:, :, None] * mean + 1e-30
        assert (np.abs(loop.out.double().cpu().numpy() - want) <= tol).all()
        ruled, size = ref.logit_rules(loop.logits.double().cpu().numpy(), [0, 1, 2], tokens=[t + [0] for t in text], n_tokens=[step, step], repetition=[float(np.float32(1.2)), 1.5],
                                      frequency=[0.5, 0.25])
        assert (np.abs(loop.ruled.double().cpu().numpy() - ruled) <= 5 * U * size).all()
        for r in range(2):
            token, lp, border = ref.sample(loop.ruled[r].double().cpu().numpy(), float(loop.uniform[r]), **{n: t[r].item() for n, t in loop.filters.items()})
            assert int(loop.token[r]) == token or border < 2.0 ** -27
            assert abs(float(loop.logprob[r]) - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -26 or border < 2.0 ** -27
        loop.after(step)


@pytest.mark.parametrize("dtype,cache", [(torch.float32, torch.int8), (torch.bfloat16, torch.float8_e4m3fn)], ids=str)
def test_a_captured_step_replays_on_new_lengths(dtype, cache):
    eager, graphed = Loop(dtype, cache, 2), Loop(dtype, cache, 2)
    eager.inputs(0), graphed.inputs(0)
    want = eager.step(0)
    graphed.calls()                                               # (warm; the same again under the capture's replay)
    before = [t.clone() for t in (graphed.kc.view(torch.uint8), graphed.vc.view(torch.uint8), graphed.ks, graphed.vs)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graphed.calls()
    for step in range(1, 40):                                     # past blocks, pages, parts and the window
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, graphed.results()):
            assert torch.equal(a, b)
        graphed.after(step - 1)
        eager.inputs(step), graphed.inputs(step)                  # eager work of the program between the replays
        want = eager.step(step)
    assert any(not torch.equal(a, b) for a, b in zip(before, (graphed.kc.view(torch.uint8), graphed.vc.view(torch.uint8), graphed.ks, graphed.vs)))


def test_two_loops_on_two_streams():
    make = lambda: (Loop(torch.float32, torch.int8, 3), Loop(torch.bfloat16, torch.float8_e4m3fn, 4))
    a, b = make()
    a2, b2 = make()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got, want = [], []
    for step in range(12):
        with torch.cuda.stream(s1):
            a.inputs(step)
            x = a.step(step)
        with torch.cuda.stream(s2):
            b.inputs(step)
            y = b.step(step)
        got.append((x, y))
    torch.cuda.synchronize()
    for step in range(12):
        a2.inputs(step), b2.inputs(step)
        want.append((a2.step(step), b2.step(step)))
    for g, w in zip(got, want):
        for x, y in zip(g, w):
            assert all(torch.equal(p, q) for p, q in zip(x, y))


@pytest.mark.parametrize("cache", [torch.float8_e4m3fn, torch.int8], ids=str)
def test_a_prompt_at_once_or_in_pieces(cache):
    """Codes depend on how tokens arrive only where a block's scale grew: a prompt whose blocks arrive whole is the same in one call and in several, and its attention is too."""
    p = pkg()
    gen = torch.Generator(device=DEV).manual_seed(6)
    n, cuts = 300, [0, 64, 160, 300]
    q, k, v = (torch.randn(n, h, D, device=DEV, generator=gen).bfloat16() for h in (H, KVH, KVH))
    table = i32([list(range(10))[::-1]])
    got = []
    for pieces in ([0, n], cuts):
        kc, vc = (torch.zeros(10, KVH, PAGE, D, dtype=torch.int8, device=DEV).view(cache) for _ in range(2))
        ks, vs = (torch.zeros(10, KVH, 2, device=DEV) for _ in range(2))
        kv, outs = p.PagedKV8(kc, vc, table, ks, vs), []
        for a, b in zip(pieces, pieces[1:]):
            c = p.Chunk(i32([0, b - a]), i32([b]), b - a, b - a, b)
            qr = torch.empty_like(q[a:b])
            p.rope(p.rope_plan(D), q[a:b], k[a:b], v[a:b], chunk=c, kv=kv, q_out=qr)
            outs.append(p.chunk_attention(qr, kv, c))
        got.append((kc.view(torch.uint8), vc.view(torch.uint8), ks, vs, torch.cat(outs)))
    for a, b in zip(got[0][:4], got[1][:4]):
        assert torch.equal(a, b)
    x, y = got[0][4].float(), got[1][4].float()                   # (parts are joined in another order: a weight's rounding apart)
    assert ((x - y).abs() <= 2.0 ** -7 * (y.abs() + v.float().abs().amax())).all()
