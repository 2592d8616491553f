"""Penalties, biases and masks on logits against the oracle in 64 bits.

Tolerances.  u = 2^-24: a quotient or product, the penalty's product and sum, its subtraction and the bias round once each: 5 u of the sum of absolute values on
the way.  bf16 logits round once more, by 2^-8 of the value at most."""
import numpy as np
import pytest
import torch

from oracle import operators as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def pkg():
    import paper_2401_15077_amd
    return paper_2401_15077_amd


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def words(bits):
    """[rows, V] truth values -> int32 words, a bit a token."""
    R, V = bits.shape
    pad = np.zeros((R, -(-V // 32) * 32), np.int64)
    pad[:, :V] = bits
    w = (pad.reshape(R, -1, 32) << np.arange(32)).sum(-1)
    return np.where(w >= 2 ** 31, w - 2 ** 32, w).astype(np.int32)


def check(got, want, size, dtype):
    got = got.double().cpu().numpy()
    fin = np.isfinite(want)
    np.testing.assert_array_equal(got[~fin], want[~fin])
    tol = 5 * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) * 1.001 if dtype == torch.bfloat16 else 0.0)
    bad = np.abs(got[fin] - want[fin]) > tol[fin]
    assert not bad.any(), (np.argwhere(bad)[:5], got[fin][bad][:5], want[fin][bad][:5])


@pytest.mark.parametrize("vocab", [2, 31, 1000, 1024, 4099, 40001])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("what", ["all", "penalties", "bias", "mask", "nothing"])
def test_rules(vocab, dtype, what):
    p = pkg()
    rng = np.random.default_rng(vocab)
    counts = [1, 3, 0, 2]
    start = np.cumsum([0] + counts)
    R, S = start[-1], len(counts)
    longest = 700
    tokens = (rng.random((S, longest)) ** 4 * vocab).astype(np.int64)
    tokens[:, 5] = [-1, vocab, 2 ** 31 - 1, -2 ** 31]                # ids outside the vocabulary count for nothing
    n_tokens, n_prompt = [0, 1, 50, longest + 100], [0, 5, 20, 333]  # (more than there are: not read)
    rep, pres, freq = np.float32([1.3, 0.8, 1.0, 2.5]), np.float32([0.5, 0.0, -0.3, 0.1]), np.float32([0.2, 0.7, 0.0, 0.05])
    masks = np.array([0b1, 0b1, 0b11, 0b101, 0b1, 0b11], np.int64)
    path = rng.integers(0, vocab, R)
    path[3] = path[1]                                                # a token twice on a path
    bstart = np.array([0, 4, 4, 5, 8])
    btoken = np.array([0, vocab - 1, 0, vocab, 3 % vocab, 1, 1, 1])   # the last of several entries counts; one is outside
    bvalue = np.float32([1.0, -2.0, 5.0, 9.0, 1.5, 1.0, 2.0, -3.0])
    bits = rng.random((3, vocab)) < 0.3
    bits[1] = False                                                  # a mask that leaves nothing
    arow = np.array([0, 1, 2, -1, 3, 0])                              # no mask: -1, and beyond the last
    x = torch.randn(int(R), vocab, device=DEV, generator=torch.Generator(device=DEV).manual_seed(vocab)).mul_(3).to(TYPES[dtype])
    x[0, 0], x[1, vocab - 1] = float("inf"), float("-inf")
    kw, call = {}, {}
    if what in ("all", "penalties"):
        kw = dict(tokens=tokens, n_tokens=np.minimum(n_tokens, longest), n_prompt=n_prompt, repetition=rep, presence=pres, frequency=freq)
        call = dict(path_token=path, path_mask=masks)
    if what in ("all", "bias"):
        kw["bias"] = (bstart, btoken, bvalue)
    if what in ("all", "mask"):
        call.update(allowed=words(bits), allowed_row=arow)
    f32 = lambda a: torch.tensor(a, device=DEV)
    rules = p.LogitRules(i32(tokens) if "tokens" in kw else None, i32(n_tokens) if "tokens" in kw else None, n_seqs=S, n_prompt=i32(n_prompt) if "tokens" in kw else None,
                         repetition=f32(rep) if "tokens" in kw else None, presence=f32(pres) if "tokens" in kw else None, frequency=f32(freq) if "tokens" in kw else None,
                         bias=(i32(bstart), i32(btoken), f32(bvalue)) if "bias" in kw else None)
    dev_call = {n: (torch.tensor(a, dtype=torch.int64 if n == "path_mask" else torch.int32, device=DEV)) for n, a in call.items()}
    out = torch.full_like(x, 5.0)
    p.apply_logit_rules(x, rules, row_start=i32(start), out=out, **dev_call)
    want, size = ref.logit_rules(x.double().cpu().numpy(), start, **kw, **call)
    check(out, want, size, x.dtype)
    # in place, and with rows that start anywhere: the same bits
    y = x.clone()
    p.apply_logit_rules(y, rules, row_start=i32(start), **dev_call)
    assert torch.equal(y, out)
    store = torch.full((int(R) * (vocab + 5) + 3,), 2.0, dtype=x.dtype, device=DEV)
    odd = store[3:].view(int(R), vocab + 5)[:, 1:vocab + 1]
    odd.copy_(x)
    other = torch.full((int(R), vocab + 3), 2.0, dtype=x.dtype, device=DEV)
    p.apply_logit_rules(odd, rules, row_start=i32(start), out=other[:, 2:vocab + 2], **dev_call)
    assert torch.equal(other[:, 2:vocab + 2], out) and torch.all(other[:, :2] == 2.0) and torch.all(other[:, vocab + 2:] == 2.0)
    p.apply_logit_rules(odd, rules, row_start=i32(start), **dev_call)
    assert torch.equal(odd, out)
    assert float(store[:3].sum()) == 6.0 and torch.all(store[3:].view(int(R), -1)[:, vocab + 1:] == 2.0) and torch.all(store[3:].view(int(R), -1)[:, :1] == 2.0)


def test_one_row_a_sequence_and_rows_of_none():
    p = pkg()
    V = 100
    x = torch.randn(3, V, device=DEV)
    rules = p.LogitRules(i32([[1, 1], [2, 3], [4, 4]]), i32([2, 2, 2]), frequency=torch.tensor([1.0, 1.0, 1.0], device=DEV))
    want = x.clone()
    want[0, 1] -= 2
    want[1, 2] -= 1
    want[1, 3] -= 1
    want[2, 4] -= 2
    out = torch.empty_like(x)
    p.apply_logit_rules(x, rules, out=out)
    assert torch.equal(out, want)
    # rows 0 and 4 belong to no sequence
    y = torch.randn(5, V, device=DEV)
    out = torch.full_like(y, 8.0)
    p.apply_logit_rules(y, rules, row_start=i32([1, 2, 2, 4]), out=out)
    want = torch.full_like(y, 8.0)
    want[1:4] = y[1:4]
    want[1, 1] -= 2
    want[2:4, 4] -= 2
    assert torch.equal(out, want)
    # a repetition that is not above 0 counts as 1; NaN logits stay NaN
    y = torch.randn(3, V, device=DEV)
    y[0, 1] = float("nan")
    r2 = p.LogitRules(i32([[1, 1], [2, 3], [4, 4]]), i32([2, 2, 2]), repetition=torch.tensor([2.0, 0.0, float("nan")], device=DEV))
    z = p.apply_logit_rules(y.clone(), r2)
    assert torch.isnan(z[0, 1]) and torch.equal(z[1:], y[1:])
    p.apply_logit_rules(y[:0], r2, row_start=i32([0, 0, 0, 0]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("repeated", [False, True])
def test_long_lists(dtype, repeated):
    """More entries and more text than a work-group has threads, from lists that start anywhere; entries for a token again, thousands later."""
    p = pkg()
    rng = np.random.default_rng(5 + repeated)
    S, V, longest = 3, 5003, 9001
    tokens = rng.integers(0, V, (S, longest))
    n_tokens, n_prompt = [longest, 8193, 4099], [17, 8200, 0]
    counts = [4000, 1, 2500]
    bstart = np.cumsum([0] + counts)
    btoken = np.concatenate([rng.integers(0, V, n) if repeated else rng.permutation(V)[:n] for n in counts])
    bvalue = rng.standard_normal(bstart[-1]).astype(np.float32)
    pres, freq, rep = np.float32([0.5, 0.0, -0.3]), np.float32([0.2, 0.7, 0.0]), np.float32([1.3, 3.0, 0.7])
    x = torch.randn(S, V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).mul_(3).to(TYPES[dtype])
    f32 = lambda a: torch.tensor(a, device=DEV)
    wide = i32(np.concatenate([np.zeros((S, 1)), tokens, np.zeros((S, 1))], 1))
    rules = p.LogitRules(wide[:, 1:-1], i32(n_tokens), n_prompt=i32(n_prompt), repetition=f32(rep), presence=f32(pres), frequency=f32(freq),
                         bias=(i32(bstart), i32(btoken), f32(bvalue)))
    want, size = ref.logit_rules(x.double().cpu().numpy(), np.arange(S + 1), tokens=tokens, n_tokens=n_tokens, n_prompt=n_prompt, repetition=rep, presence=pres, frequency=freq,
                                 bias=(bstart, btoken, bvalue))
    check(p.apply_logit_rules(x, rules, out=torch.empty_like(x)), want, size, x.dtype)


def test_texts_that_are_views():
    """What a sequence says beyond its columns is not read, and one text may stand for all sequences."""
    p = pkg()
    V = 64
    wide = i32(np.arange(60).reshape(3, 20))
    x = torch.zeros(3, V, device=DEV)
    ones = torch.ones(3, device=DEV)
    y = p.apply_logit_rules(x.clone(), p.LogitRules(wide[:, 2:7], i32([3, 50, 2 ** 31 - 1]), frequency=ones))
    want = torch.zeros_like(x)
    for s, n in enumerate([3, 5, 5]):
        want[s, 20 * s + 2:20 * s + 2 + n] = -1
    assert torch.equal(y, want)
    y = p.apply_logit_rules(x.clone(), p.LogitRules(wide[1:2, :6].expand(3, 6), i32([1, -4, 6]), frequency=ones))
    want.zero_()
    want[0, 20] = -1
    want[2, 20:26] = -1
    assert torch.equal(y, want)


def test_a_long_text_of_one_token_counts_exactly():
    p = pkg()
    n = 200000
    x = torch.zeros(1, 50, device=DEV)
    rules = p.LogitRules(torch.full((1, n), 7, dtype=torch.int32, device=DEV), i32([n]), n_prompt=i32([1000]), frequency=torch.tensor([1.0], device=DEV))
    assert float(p.apply_logit_rules(x, rules)[0, 7]) == -(n - 1000.0)
