"""More sequences than a wave has lanes: the owner of a row is found over several rounds of 64 boundaries.  Bounds as in the operators' own tests: a rotation 8 u of what it adds up, a score 64 u of
scale * sum |q k| (twice in a weight) and 64 u for the sums, a rule 5 u of what it adds up; u = 2^-24."""
import numpy as np
import pytest
import torch

from oracle import operators as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
SEQUENCES = [63, 64, 65, 128, 129, 200]


def pkg():
    import paper_2401_15077_amd
    return paper_2401_15077_amd


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def batch(S, longest, seed):
    """0 to 3 rows a sequence, the last with one at least; keys of their own length; two rows in front of the first sequence and one behind the last."""
    rng = np.random.default_rng(seed)
    rows = rng.integers(0, 4, S)
    rows[-1] = max(1, rows[-1])
    keys = rows + rng.integers(0, longest, S)
    start = 2 + np.cumsum(np.concatenate([[0], rows]))
    return rows, keys, start, int(start[-1]) + 1


@pytest.mark.parametrize("S", SEQUENCES)
def test_rotation_and_append(S):
    p = pkg()
    rows, keys, start, R = batch(S, 40, S)
    KVH, D, page = 1, 16, 8
    gen = torch.Generator(device=DEV).manual_seed(S)
    q, k, v = (torch.randn(R, KVH, D, device=DEV, generator=gen) for _ in range(3))
    per = int(-(-max(keys) // page))
    table = np.random.default_rng(S).permutation(S * per).reshape(S, per)
    kc, vc = torch.zeros(S * per, KVH, page, D, device=DEV), torch.zeros(S * per, KVH, page, D, device=DEV)
    q_out = torch.full_like(q, 7.0)
    p.rope(p.rope_plan(D), q, k, v, chunk=p.Chunk(i32(start), i32(keys), R, 3, int(max(keys)) + 1), kv=p.PagedKV(kc, vc, i32(table)), q_out=q_out)
    facts = ref.chunk_rows(start, keys)
    pos = np.zeros(R)
    want_k, want_v = np.zeros(kc.shape), np.zeros(vc.shape)
    owned = np.zeros(R, bool)
    for r, s, t, at, _ in facts:
        pos[r], owned[r] = at, True
    f = ref.frequencies(D)
    (wq, size), (wk, ksize) = (ref.rotate(x.cpu().numpy(), pos, f, D, False) for x in (q, k))
    tol = np.zeros(kc.shape)
    for r, s, t, _, _ in facts:
        cell = table[s, t // page], slice(None), t % page
        want_k[cell], want_v[cell], tol[cell] = wk[r], v[r].cpu().numpy(), 8 * U * ksize[r]
    got = q_out.double().cpu().numpy()
    assert (np.abs(got - wq)[owned] <= 8 * U * size[owned]).all() and (got[~owned] == 7.0).all() and (~owned).sum() == 3
    assert (np.abs(kc.double().cpu().numpy() - want_k) <= tol).all() and (vc.double().cpu().numpy() == want_v).all()


@pytest.mark.parametrize("S", SEQUENCES)
@pytest.mark.parametrize("longest", [30, 400])                    # one part, and parts that are joined
def test_attention(S, longest):
    p = pkg()
    rows, keys, start, R = batch(S, longest, S + 1)
    H, KVH, D, page = 2, 1, 32, 16
    gen = torch.Generator(device=DEV).manual_seed(S)
    per = int(-(-max(keys) // page))
    table = np.random.default_rng(S).permutation(S * per).reshape(S, per)
    kc, vc = (torch.randn(S * per, KVH, page, D, device=DEV, generator=gen) for _ in range(2))
    q = torch.randn(R, H, D, device=DEV, generator=gen)
    out = torch.full_like(q, 7.0)
    chunk, kv = p.Chunk(i32(start), i32(keys), R, 3, int(max(keys))), p.PagedKV(kc, vc, i32(table))
    assert (p.chunk_attention_workspace(q, kv, chunk) > 256) == (longest == 400)
    p.chunk_attention(q, kv, chunk, out=out)
    want, mean, big, count = ref.attention(q.double().cpu().numpy(), kc.double().cpu().numpy(), vc.double().cpu().numpy(), table, ref.chunk_rows(start, keys), R, keys, page=page,
                                           scale=D ** -0.5)
    got = out.double().cpu().numpy()
    owned = ~np.isnan(want[:, 0, 0])
    assert (got[~owned] == 7.0).all() and (~owned).sum() == 3
    tol = (2 * 64 * U * big + 64 * U)[:, :, None] * mean
    assert (np.abs(got - want)[owned] <= tol[owned]).all()


@pytest.mark.parametrize("S", SEQUENCES)
def test_logit_rules(S):
    p = pkg()
    rows, _, start, R = batch(S, 1, S + 2)
    V, longest = 300, 20
    rng = np.random.default_rng(S)
    tokens, n_tokens, n_prompt = rng.integers(0, V, (S, longest)), rng.integers(0, longest + 1, S), rng.integers(0, 10, S)
    rep, pres, freq = (rng.random(S).astype(np.float32) + 0.5 for _ in range(3))
    bstart = np.arange(S + 1) * 2
    btoken, bvalue = rng.integers(0, V, 2 * S), rng.standard_normal(2 * S).astype(np.float32)
    x = torch.randn(R, V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(S))
    f = lambda a: torch.tensor(a, device=DEV)
    rules = p.LogitRules(i32(tokens), i32(n_tokens), n_prompt=i32(n_prompt), repetition=f(rep), presence=f(pres), frequency=f(freq), bias=(i32(bstart), i32(btoken), f(bvalue)))
    out = torch.full_like(x, 7.0)
    p.apply_logit_rules(x, rules, row_start=i32(start), out=out)
    want, size = ref.logit_rules(x.cpu().numpy(), start, tokens=tokens, n_tokens=n_tokens, n_prompt=n_prompt, repetition=rep, presence=pres, frequency=freq, bias=(bstart, btoken, bvalue))
    got = out.double().cpu().numpy()
    own = slice(2, R - 1)
    assert (np.abs(got - want)[own] <= 5 * U * size[own]).all() and (got[:2] == 7.0).all() and (got[-1] == 7.0).all()
