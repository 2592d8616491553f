"""The operators beside autograd (no GPU needed: the call into the library is left out): what requires gradients is refused, and what a call writes counts as written."""
from types import SimpleNamespace

import pytest
import torch

import paper_2401_15077_amd as pkg
from paper_2401_15077_amd import operators as ops

R, S, H, KVH, D, V = 4, 2, 4, 2, 64, 50


def i32(*a):
    return torch.tensor(a, dtype=torch.int32)


def f32(*shape):
    return torch.zeros(*shape)


@pytest.fixture(autouse=True)
def no_launch(monkeypatch):
    monkeypatch.setattr(ops, "_call", lambda fn, device, *args: None)


def chunk():
    return pkg.Chunk(i32(0, 2, 4), i32(5, 6), R, 2, 10)


def cache(k=None, v=None):
    return pkg.PagedKV(f32(9, KVH, 32, D) if k is None else k, f32(9, KVH, 32, D) if v is None else v, torch.zeros(S, 4, dtype=torch.int32))


def attend(kv=None, **kw):
    return pkg.chunk_attention(kw.pop("q", f32(R, H, D)), kv or cache(), chunk(), workspace=torch.zeros(1 << 20, dtype=torch.uint8), **kw)


def turn(kv=None, **kw):
    pkg.rope(pkg.rope_plan(D), kw.pop("q", f32(R, H, D)), kw.pop("k", f32(R, KVH, D)), f32(R, KVH, D) if kv is not None else None, chunk=chunk(), kv=kv, **kw)


def rule(rules=None, **kw):
    return pkg.apply_logit_rules(kw.pop("logits", f32(R, V)), rules or pkg.LogitRules(n_seqs=S), row_start=i32(0, 2, 4), **kw)


def rules(**kw):
    return pkg.LogitRules(n_seqs=S, repetition=f32(S), **kw)


def biased(value):
    return pkg.LogitRules(n_seqs=S, bias=(i32(0, 1, 2), i32(3, 4), value))


CALLS = {
    "k of the cache, read": lambda t: attend(cache(k=t(9, KVH, 32, D))), "v of the cache, read": lambda t: attend(cache(v=t(9, KVH, 32, D))),
    "k of the cache, written": lambda t: turn(cache(k=t(9, KVH, 32, D))), "v of the cache, written": lambda t: turn(cache(v=t(9, KVH, 32, D))),
    "slopes": lambda t: attend(slopes=t(H)), "out of the attention": lambda t: attend(out=t(R, H, D)), "q": lambda t: attend(q=t(R, H, D)),
    "q_out": lambda t: turn(cache(), q_out=t(R, H, D)), "k_out": lambda t: turn(k_out=t(R, KVH, D)),
    "logits": lambda t: rule(logits=t(R, V)), "out of the rules": lambda t: rule(out=t(R, V)),
    "presence": lambda t: rule(rules(presence=t(S))), "frequency": lambda t: rule(rules(frequency=t(S))), "bias value": lambda t: rule(biased(t(2))),
}


def leaf(*shape):
    return torch.zeros(*shape, requires_grad=True)


@pytest.mark.parametrize("name", CALLS)
def test_what_requires_gradients_is_refused(name):
    with pytest.raises(ValueError, match="requires gradients"):
        CALLS[name](leaf)
    CALLS[name](lambda *shape: leaf(*shape).detach())
    with torch.no_grad():
        CALLS[name](leaf)


def test_rules_that_were_made_while_gradients_were_off():
    with torch.no_grad():
        made = rules(presence=leaf(S))
        rule(made)
    with pytest.raises(ValueError, match="presence requires gradients"):
        rule(made)


def test_context_setters():
    c = SimpleNamespace(torch=torch, device=torch.device("cpu"), max_batch=2, M=3, shape=SimpleNamespace(vocab=V, n_heads=H), lib=None, h=None)
    with pytest.raises(ValueError, match="slopes requires gradients"):
        pkg.Eagle.set_attention(c, slopes=leaf(H))
    with pytest.raises(ValueError, match="frequency requires gradients"):
        pkg.Eagle.set_logit_rules(c, frequency=leaf(2))


def test_what_a_call_writes_counts_as_written():
    """And nothing else does."""
    def versions(call, **named):
        before = {n: t._version for n, t in named.items()}
        call()
        return {n for n, t in named.items() if t._version != before[n]}

    q, k, v, q2, k2, kc, vc, x, y = f32(R, H, D), f32(R, KVH, D), f32(R, KVH, D), f32(R, H, D), f32(R, KVH, D), f32(9, KVH, 32, D), f32(9, KVH, 32, D), f32(R, V), f32(R, V)
    plan, c, kv = pkg.rope_plan(D), chunk(), cache(kc, vc)
    every = dict(q=q, k=k, v=v, q2=q2, k2=k2, kc=kc, vc=vc, x=x, y=y)
    assert versions(lambda: pkg.rope(plan, q, k, v, chunk=c, kv=kv), **every) == {"q", "kc", "vc"}
    assert versions(lambda: pkg.rope(plan, q, k, chunk=c, kv=kv, q_out=q2), **every) == {"q2", "kc"}
    assert versions(lambda: pkg.rope(plan, None, k, v, chunk=c, kv=kv), **every) == {"kc", "vc"}
    assert versions(lambda: pkg.rope(plan, q, k, chunk=c, q_out=q2, k_out=k2), **every) == {"q2", "k2"}
    assert versions(lambda: pkg.rope(plan, None, k, chunk=c), **every) == {"k"}
    assert versions(lambda: pkg.rope(plan, q, None, chunk=c), **every) == {"q"}
    assert versions(lambda: attend(kv, q=q, out=q2), **every) == {"q2"}
    assert versions(lambda: attend(kv, q=q, out=q), **every) == {"q"}
    assert versions(lambda: rule(logits=x, out=y), **every) == {"y"}
    assert versions(lambda: rule(logits=x), **every) == {"x"}


def test_a_saved_tensor_that_a_call_overwrites_is_noticed():
    w = leaf(R, V)
    x = w * 2.0
    loss = (x * x).sum()                                          # saves x
    rule(logits=x.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_tensors_of_inference_mode():
    with torch.inference_mode():
        x = f32(R, V)
        rule(logits=x)
        attend(q=f32(R, H, D))
        turn(cache())
