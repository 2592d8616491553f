"""Steps of a context with other positions, ruled attention and ruled logits (eagle_set_rope, eagle_set_attention, eagle_set_logit_rules), in lock-step with the oracle.
The tolerances are those of the plain steps (tests/test_gpu_parity.py): positions and masks change which numbers are added up, not how; the penalties scale a logit by at most
1.3 here, their own roundings are 2^-24 of it."""
import math

import numpy as np
import pytest
import torch

import paper_2401_15077_amd as pkg
import synth
from lockstep import Stats, check_prefill, lockstep_step, lockstep_step_batch
from oracle import operators as ref
from oracle.eagle_oracle import Oracle, rmsnorm, round_bf16, softmax

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = {"fp32": 1e-4, "bf16": 2e-2}


class Ruled(Oracle):
    """The oracle's model with the definitions of oracle/operators.py in place of its own positions, scores and logits."""
    rope_kw, mscale, interleaved, rot = None, 1.0, False, 0
    softcap, window, slopes = 0.0, 0, None
    rules = None                                                  # keywords of ref.logit_rules by slot, without texts
    mask_of = None                                                # node -> row of `allowed`

    def _turn(self, x, pos):
        s = self.s
        if self.rope_kw is None:
            from oracle.eagle_oracle import rope
            return rope(x, pos, s.rope_theta)
        return ref.rotate(x, pos, ref.frequencies(self.rot, theta=s.rope_theta, **self.rope_kw), self.rot, self.interleaved, self.mscale)[0].astype(x.dtype)

    def _layer(self, prefix, h, pos, kc, vc, slots, visible, moe, stage_key):
        s, R = self.s, h.shape[0]
        x = rmsnorm(h, self._lw(prefix, "attn_norm"), s.rms_eps)
        q = self._turn((x @ self._lw(prefix, "wq").T).reshape(R, s.n_heads, s.head_dim), pos)
        k = self._turn((x @ self._lw(prefix, "wk").T).reshape(R, s.n_kv_heads, s.head_dim), pos)
        v = (x @ self._lw(prefix, "wv").T).reshape(R, s.n_kv_heads, s.head_dim)
        kc[slots] = round_bf16(k) if self.kv_store == "bf16" else k
        vc[slots] = round_bf16(v) if self.kv_store == "bf16" else v
        Tn, g = visible.shape[1], s.n_heads // s.n_kv_heads
        # the tokens that a row sees lie on its path, one position apart: their order among them is their position
        dist = (visible.sum(1)[:, None] - 1) - (np.cumsum(visible, axis=1) - 1)
        seen = visible & (dist < self.window) if self.window else visible
        att = np.empty((R, s.n_heads, s.head_dim), dtype=h.dtype)
        for hd in range(s.n_heads):
            sc = (q[:, hd, :] @ kc[:Tn, hd // g, :].T) / math.sqrt(s.head_dim)
            if self.softcap:
                sc = self.softcap * np.tanh(sc / self.softcap)
            if self.slopes is not None:
                sc = sc - self.slopes[hd] * dist
            att[:, hd, :] = softmax(np.where(seen, sc, -np.inf)) @ vc[:Tn, hd // g, :]
        h = h + att.reshape(R, -1) @ self._lw(prefix, "wo").T
        return h + self._mlp(prefix, rmsnorm(h, self._lw(prefix, "mlp_norm"), s.rms_eps), moe, stage_key)

    def _target_forward(self, toks, pos, slots, visible, stage):
        F, L = super()._target_forward(toks, pos, slots, visible, stage)
        if self.rules is None:
            return F, L
        L = L.copy()
        rows = [len(toks) - 1] if stage == "prefill" else range(len(toks))
        if stage == "prefill":
            self.n_prompt = len(toks)
        for r in rows:
            text = list(toks) if stage == "prefill" else list(self.x)
            node = 0
            if stage == "verify":
                node = r
                text += [self.tok[u] for u in self.tree.ancestors_or_self(r) if u != 0]
            kw = dict(self.rules)
            if "allowed" in kw:
                kw["allowed_row"] = [self.mask_of[node]]
            L[r] = ref.logit_rules(L[r:r + 1], [0, 1], tokens=[text], n_tokens=[len(text)], n_prompt=[self.n_prompt], **kw)[0]
        return F, L


def pair(shape, tree, seed, *, temperature=0.0, kv="fp32", max_batch=1, max_seq=256, rope=None, attn=None, slots=1, **kw):
    s = synth.SHAPES[shape]
    par, rk = synth.TREES[tree]
    eng = pkg.Eagle(s, par, rk, max_seq=max_seq, temperature=temperature, seed=7, kv_dtype=kv, max_batch=max_batch, **kw)
    if rope is not None:
        eng.set_rope(**rope)
    eng.load_weights(synth.iter_weights(s, seed, synth.device_fmt(s)))
    W = synth.make_weights(s, seed, synth.oracle_fmt(s))
    orcs = []
    slopes = None
    if attn is not None:
        a = dict(attn)
        if a.pop("slopes", False):
            slopes = torch.tensor(2.0 ** (-4.0 * np.arange(1, s.n_heads + 1) / s.n_heads), dtype=torch.float32, device=DEV)
        eng.set_attention(slopes=slopes, **a)
    for b in range(slots):
        o = Ruled(s, W, par, rk, max_seq=max_seq, temperature=temperature, seed=7, seq_id=b, kv_store="bf16" if kv == "bf16" else None)
        if rope is not None:
            r = dict(rope)
            o.rot, o.interleaved, o.mscale = r.pop("rot_dim", s.head_dim), r.pop("interleaved", False), r.pop("mscale", 1.0)
            o.rope_kw = r
        if attn is not None:
            o.softcap, o.window = attn.get("softcap", 0.0), attn.get("window", 0)
            o.slopes = None if slopes is None else slopes.double().cpu().numpy()
        orcs.append(o)
    return s, eng, orcs


ROPES = [dict(scaling="linear", factor=4.0), dict(interleaved=True), dict(rot_dim=32, scaling="ramp", factor=8.0, low=1.0, high=32.0, trained_len=64, mscale=1.2),
         dict(rot_dim=16, interleaved=True, scaling="bands", factor=4.0, trained_len=64)]


@pytest.mark.parametrize("rope", ROPES, ids=str)
@pytest.mark.parametrize("shape,kv", [("tiny", "fp32"), ("mini-gqa", "fp32")])
def test_positions(shape, kv, rope):
    rope = dict(rope)
    if shape == "mini-gqa" and rope.get("rot_dim") == 32:
        rope["rot_dim"] = 20                                      # (heads of 32)
    s, eng, (orc,) = pair(shape, "T15", 3, rope=rope, kv=kv)
    tol = TOL[s.dtype]
    prompt = synth.prompt(3, 40, s.vocab)
    check_prefill(eng, orc, prompt, tol)
    st = Stats()
    for _ in range(4):
        lockstep_step(eng, orc, st, tol)
    # keys come back in the model's own order of elements
    for layer, kc in ((0, orc.kc[0]), (s.n_layers - 1, orc.kc[-1]), (pkg.HEAD_LAYER, orc.dkc)):
        for pos in (0, 17, 39):
            k, _ = eng.get_kv_row(0, layer, pos)
            assert np.abs(k - kc[pos].reshape(-1)).max() < (1e-4 if s.dtype == "fp32" else 2e-2)
    with pytest.raises(pkg.EagleError, match="before"):
        eng.set_rope(interleaved=True)
    eng.close()


ATTENTIONS = [dict(softcap=2.0), dict(window=9), dict(slopes=True), dict(softcap=3.0, window=30, slopes=True)]


@pytest.mark.parametrize("shape,kv,attn", [(sh, kv, a) for sh, kv in (("tiny", "fp32"), ("tiny", "bf16"), ("mini-gqa", "fp32")) for a in ATTENTIONS] + [("mini-moe", "fp32", dict(window=9))], ids=str)
def test_attention(shape, kv, attn):
    s, eng, (orc,) = pair(shape, "T26", 4, attn=attn, kv=kv)
    tol = TOL["bf16"] if kv == "bf16" else TOL[s.dtype]
    prompt = synth.prompt(4, 45, s.vocab)
    check_prefill(eng, orc, prompt, tol)
    st = Stats()
    for _ in range(4):
        lockstep_step(eng, orc, st, tol)
    with pytest.raises(pkg.EagleError, match="active"):
        eng.set_attention(window=3)
    # vanilla steps, and plain attention again
    orc2 = orc
    eng.vanilla_step()
    orc2.vanilla_step()
    assert np.abs(eng.get_buffer(pkg.BUF_VANILLA_LOGITS) - orc2.vanilla_logits).max() <= tol
    eng.reset()
    eng.set_attention()
    plain = Oracle(s, synth.make_weights(s, 4, synth.oracle_fmt(s)), *synth.TREES["T26"], max_seq=256, seed=7, kv_store="bf16" if kv == "bf16" else None)
    check_prefill(eng, plain, prompt, tol)
    st = Stats()
    lockstep_step(eng, plain, st, tol)
    eng.close()


def test_ruled_attention_over_long_prompts_and_batches():
    """Prompts of several passes (512-row windows of the bf16 models), batches of more than 32 rows, and both caches of a 33-row pass."""
    s, eng, orcs = pair("mini-gqa", "T15", 5, attn=dict(softcap=4.0, window=100, slopes=True), max_batch=4, max_seq=700, slots=4)
    sts = [Stats() for _ in orcs]
    for b, o in enumerate(orcs):
        check_prefill(eng, o, synth.prompt(5, [600, 40, 7, 200][b], s.vocab, stream=b), TOL["bf16"], seq=b)
    for _ in range(2):
        lockstep_step_batch(eng, orcs, sts, TOL["bf16"])
    eng.close()


def rules_for(V, M, B, rng):
    bits = rng.random((3, V)) < 0.5
    pad = np.zeros((3, -(-V // 32) * 32), np.int64)
    pad[:, :V] = bits
    w = (pad.reshape(3, -1, 32) << np.arange(32)).sum(-1)
    words = np.where(w >= 2 ** 31, w - 2 ** 32, w).astype(np.int32)
    per = [dict(repetition=[1.0 + 0.3 * rng.random()], presence=[0.3 * rng.random()], frequency=[0.2 * rng.random()]) for _ in range(B)]
    for p in per:
        for k in p:
            p[k] = [float(np.float32(p[k][0]))]
    bias = [(rng.permutation(V)[:5], np.float32(rng.standard_normal(5))) for _ in range(B)]
    return bits, words, per, bias


@pytest.mark.parametrize("temperature", [0.0, 1.0])
@pytest.mark.parametrize("shape,slots", [("tiny", 1), ("mini-gqa", 3)])
def test_logit_rules(shape, slots, temperature):
    """Penalties along the paths, biases and masks a node (rewritten between steps), greedy and sampled; what is masked is never emitted."""
    s, eng, orcs = pair(shape, "T15", 6, temperature=temperature, max_batch=slots, slots=slots)
    tol = TOL[s.dtype]
    V, M = s.vocab, len(synth.TREES["T15"][0])
    rng = np.random.default_rng(11)
    bits, words, per, bias = rules_for(V, M, slots, rng)
    f32 = lambda name: torch.tensor([p[name][0] for p in per], dtype=torch.float32, device=DEV)
    start = np.cumsum([0] + [len(b[0]) for b in bias])
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    rows = rng.integers(-1, 3, (slots, M))
    arow = i32(rows.reshape(-1))
    eng.set_logit_rules(repetition=f32("repetition"), presence=f32("presence"), frequency=f32("frequency"),
                        bias=(i32(start), i32(np.concatenate([b[0] for b in bias])), torch.tensor(np.concatenate([b[1] for b in bias]), device=DEV)),
                        allowed=i32(words), allowed_row=arow)
    for b, o in enumerate(orcs):
        o.rules = dict(per[b], bias=([0, 5], bias[b][0], bias[b][1]), allowed=words)
        o.mask_of = rows[b]
    margin = 2e-2 if temperature == 0.0 else 5e-2
    for b, o in enumerate(orcs):
        prompt = synth.prompt(6, 30 + 5 * b, V, stream=b)
        first = eng.prefill(b, prompt)
        want = o.prefill(prompt)
        same(eng.get_buffer(pkg.BUF_VANILLA_LOGITS, b), o.prefill_logits[-1], tol)
        assert first == want or o.first_margin < margin
        o.x[-1] = first
        assert rows[b][0] < 0 or bits[rows[b][0]][first]
    for step in range(4):
        toks = eng.draft_tree()
        for b, o in enumerate(orcs):
            d = o.draft_tree(forced_tokens=toks[b])
            assert all(m[4] < margin for m in d["mismatches"])
            rows[b] = rng.integers(-1, 3, M)                      # masks that go with the drafted tokens
        arow.copy_(i32(rows.reshape(-1)))
        eng.verify()
        for b, o in enumerate(orcs):
            o.verify()
            same(eng.get_buffer(pkg.BUF_LOGITS, b), o.L, tol)
        out, lens, path = eng.accept()
        for b, o in enumerate(orcs):
            r = o.accept()
            n = int(lens[b])
            got = [int(x) for x in out[b][:n]], [int(x) for x in path[b][:n]]
            if got != (r["emitted"], r["path"]):
                assert r["margin"] < margin
            for node, t in zip(got[1], got[0]):                   # the token behind a node of the path
                assert rows[b][node] < 0 or bits[rows[b][node]][t]
            o.commit(got[1], got[0][-1])
    eng.vanilla_step()
    for b, o in enumerate(orcs):
        o.vanilla_step()
        same(eng.get_buffer(pkg.BUF_VANILLA_LOGITS, b), o.vanilla_logits, tol)
    # no rules: the target's own logits again
    eng.set_logit_rules()
    eng.reset()
    o = Oracle(s, synth.make_weights(s, 6, synth.oracle_fmt(s)), *synth.TREES["T15"], max_seq=256, temperature=temperature, seed=7)
    check_prefill(eng, o, synth.prompt(6, 30, V), tol, margin_thr=margin)
    eng.close()


def same(got, want, tol):
    fin = np.isfinite(want)
    assert np.array_equal(fin, np.isfinite(got))
    assert np.abs(got[fin] - want[fin]).max() <= tol * 1.3


def test_a_mask_that_leaves_nothing_ends_in_a_token():
    """Every node's mask is empty: the steps run on, their tokens lie in the vocabulary."""
    for shape, temperature in (("tiny", 0.0), ("tiny", 1.0), ("tiny-v40k", 1.0)):
        s, eng, _ = pair(shape, "T8", 8, temperature=temperature)
        M = len(synth.TREES["T8"][0])
        eng.set_logit_rules(allowed=torch.zeros(1, (s.vocab + 31) // 32, dtype=torch.int32, device=DEV), allowed_row=torch.zeros(M, dtype=torch.int32, device=DEV))
        first = eng.prefill(0, synth.prompt(8, 10, s.vocab))
        assert 0 <= first < s.vocab
        assert np.isneginf(eng.get_buffer(pkg.BUF_VANILLA_LOGITS)).all()
        for _ in range(2):
            out, lens, _ = eng.step()
            assert 1 <= lens[0] <= eng.D + 1 and all(0 <= t < s.vocab for t in out[0][:lens[0]])
        assert 0 <= int(eng.vanilla_step()[0]) < s.vocab
        eng.close()


def test_together_greedy_speculation_equals_plain_decoding():
    """Other positions, a window, a cap, penalties and a bias, all at once: speculative steps emit what vanilla steps emit."""
    s, eng, _ = pair("tiny", "T26", 9, rope=dict(interleaved=True, scaling="linear", factor=2.0), attn=dict(softcap=5.0, window=24))
    f = lambda v: torch.tensor([v], dtype=torch.float32, device=DEV)
    eng.set_logit_rules(repetition=f(1.2), presence=f(0.1), frequency=f(0.3), bias=(torch.tensor([0, 1], dtype=torch.int32, device=DEV), torch.tensor([5], dtype=torch.int32, device=DEV), f(0.5)))
    prompt = synth.prompt(9, 33, s.vocab)
    out, _ = eng.generate(prompt, 40)
    eng.reset()
    van = [eng.prefill(0, prompt)]
    while len(van) < 40:
        van.append(int(eng.vanilla_step()[0]))
    assert list(out) == van
    eng.close()


def test_refusals():
    s = synth.SHAPES["tiny"]
    eng = pkg.Eagle(s, *synth.TREES["T8"], max_seq=64)
    for bad in (dict(rot_dim=65), dict(rot_dim=66), dict(scaling="linear", factor=0.5), dict(theta=0.5)):
        with pytest.raises(pkg.EagleError):
            eng.set_rope(**bad)
    with pytest.raises(ValueError):
        eng.set_rope(scaling="other")
    with pytest.raises(pkg.EagleError):
        eng.set_attention(softcap=-1.0)
    with pytest.raises(pkg.EagleError):
        eng.set_attention(window=-1)
    with pytest.raises(ValueError):
        eng.set_attention(slopes=torch.zeros(3, device=DEV))
    with pytest.raises(ValueError):
        eng.set_logit_rules(repetition=torch.zeros(2, device=DEV))
    with pytest.raises(ValueError):
        eng.set_logit_rules(allowed=torch.zeros(1, 32, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        eng.set_logit_rules(allowed=torch.zeros(1, 3, dtype=torch.int32, device=DEV), allowed_row=torch.zeros(8, dtype=torch.int32, device=DEV))
    eng.set_rope()
    eng.set_attention()
    eng.set_logit_rules()
    eng.close()
