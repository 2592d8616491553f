"""Timed cases of the operators beside the decoding step: rotary positions with the append to a paged cache, attention of a chunk of new
tokens over that cache, and the rules that logits pass before a token is chosen.

Every case is a call that a serving program makes with the tensors it has in hand.  `own` chooses between the plain form (elementary torch
operations in 32 bits, angles in 64) and the library's operators; `exact` is the definition in 64 bits.  Lengths, trees and page tables are
functions of the case, values of the seed.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    def rope(name, rows, keys, heads, kv_heads, dim, dtype, cache, tree=False, layout="half", rot=0, scaling="none", factor=1.0, start=0, inverse=False):
        return {"name": name, "kind": "rope", "rows": rows, "keys": keys, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache, "tree": tree,
                "layout": layout, "rot": rot or dim, "scaling": scaling, "factor": factor, "start": start, "inverse": inverse, "page": 64}

    def attend(name, rows, keys, heads, kv_heads, dim, dtype, cache, tree=False, softcap=0.0, window=0, slopes=False, prefix=0, page=64):
        return {"name": name, "kind": "attend", "rows": rows, "keys": keys, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache, "tree": tree,
                "softcap": softcap, "window": window, "slopes": slopes, "prefix": prefix, "page": page}

    def rules(name, seqs, rows, vocab, dtype, history, prompt, masks, bias):
        return {"name": name, "kind": "rules", "seqs": seqs, "rows": rows, "vocab": vocab, "dtype": dtype, "history": history, "prompt": prompt, "masks": masks, "bias": bias}

    # rows and keys: one number a sequence, new tokens and tokens in the cache with them
    return [
        # one user, one new token, the library's default types: nothing but latency
        rope("rope-token", "1", "701", 32, 32, 128, "fp32", "fp32"),
        # four users' draft trees; half of a head rotated in adjacent pairs, positions scaled by wavelength
        rope("rope-trees", "26 26 26 26", "1526 2051 1787 2330", 32, 8, 128, "fp32", "bf16", tree=True, layout="pairs", rot=64, scaling="bands", factor=8.0),
        # chunks of five long prompts on the way into the cache, 900 000 tokens into a document
        rope("rope-chunks", "4096 2011 1 1500 583", "4096 2100 777 1500 1024", 64, 8, 128, "bf16", "bf16", scaling="ramp", factor=32.0, start=900000),
        # the way back: gradients of rotated queries and keys of one training sequence
        rope("rope-back", "2011", "2011", 64, 8, 128, "fp32", "none", scaling="linear", factor=4.0, inverse=True),
        # one user, one new token, the library's default types
        attend("attend-token", "1", "701", 32, 32, 128, "fp32", "fp32"),
        # four users' draft trees over a half-size cache: 104 rows
        attend("attend-trees", "26 26 26 26", "1526 2051 1787 2330", 32, 8, 128, "fp32", "bf16", tree=True),
        # a full serving batch, one token each, contexts of a thousand to sixteen thousand tokens
        attend("attend-batch", "1 " * 64, " ".join(str(1024 + 241 * i) for i in range(64)), 64, 8, 128, "bf16", "bf16"),
        # chunks of two prompts in the middle of a document: capped scores, a sliding window
        attend("attend-chunks", "1536 509", "7536 2509", 32, 8, 128, "bf16", "bf16", softcap=50.0, window=4096),
        # a whole prompt in 32 bits: scores that fall with distance, a prefix that everyone sees, an odd head size
        attend("attend-prompt", "2011", "2011", 32, 32, 80, "fp32", "fp32", slopes=True, prefix=100),
        # one user, one token
        rules("rules-token", 1, 1, 32000, "fp32", 300, 120, False, 5),
        # four users' draft trees under a grammar: a mask a node, penalties along each path
        rules("rules-trees", 4, 26, 32000, "fp32", 1900, 900, True, 40),
        # a serving batch, half-width logits of a large odd vocabulary, long histories
        rules("rules-batch", 160, 1, 100003, "bf16", 6000, 4000, True, 300),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "attend", "attend", "rules"])
    if kind == "rules":
        trees = rng.random() < 0.4
        seqs = _log_int(rng, 1, 6 if trees else 160)
        return {"kind": "rules", "seqs": seqs, "rows": rng.randint(2, 40) if trees else 1, "vocab": _log_int(rng, 900, 100003), "dtype": rng.choice(["fp32", "bf16"]),
                "history": _log_int(rng, 1, 6000), "prompt": _log_int(rng, 1, 3000), "masks": rng.random() < 0.6, "bias": _log_int(rng, 1, 300)}
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (64, 8), (40, 40), (8, 2), (12, 4), (5, 1)])
    dim = rng.choice([128, 128, 128, 64, 80, 32])
    dtype = rng.choice(["fp32", "bf16"])
    cache = "bf16" if dtype == "bf16" else rng.choice(["fp32", "bf16"])
    tree = rng.random() < 0.3
    if kind == "rope":
        seqs = rng.randint(1, 6)
        rows = [rng.randint(2, 64) if tree else _log_int(rng, 1, 1200) for _ in range(seqs)]
        keys = [n + (0 if rng.random() < 0.2 else _log_int(rng, 1, 2000)) for n in rows]
        scaling = rng.choice(["none", "linear", "base", "bands", "ramp"])
        layout = rng.choice(["half", "pairs"])
        inverse = not tree and rng.random() < 0.25
        return {"kind": "rope", "rows": " ".join(map(str, rows)), "keys": " ".join(map(str, keys)), "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
                "cache": "none" if inverse else cache, "tree": tree, "layout": layout, "rot": rng.choice([dim, dim, dim // 2]), "scaling": scaling,
                "factor": 1.0 if scaling == "none" else rng.uniform(1.5, 40.0), "start": 0 if tree or rng.random() < 0.5 else _log_int(rng, 1, 1000000), "inverse": inverse,
                "page": rng.choice([16, 32, 64, 128])}
    shape = "tree" if tree else rng.choice(["token", "token", "chunk"])
    seqs = {"tree": rng.randint(1, 6), "token": _log_int(rng, 1, 32), "chunk": rng.randint(1, 3)}[shape]
    rows = [{"tree": rng.randint(2, 64), "token": rng.choice([1, 1, 1, 2, 7]), "chunk": _log_int(rng, 20, 1000)}[shape] for _ in range(seqs)]
    keys = [n + (0 if rng.random() < 0.1 else _log_int(rng, 1, {"tree": 3000, "token": 6000, "chunk": 2500}[shape])) for n in rows]
    return {"kind": "attend", "rows": " ".join(map(str, rows)), "keys": " ".join(map(str, keys)), "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache,
            "tree": tree, "softcap": rng.choice([0.0, 0.0, 30.0]), "window": rng.choice([0, 0, _log_int(rng, 16, 2000)]), "slopes": rng.random() < 0.3,
            "prefix": rng.choice([0, 0, _log_int(rng, 1, 500)]), "page": rng.choice([16, 32, 64, 128])}


# ----------------------------------------------------------------------------- inputs
def _lengths(case):
    return [int(x) for x in case["rows"].split()], [int(x) for x in case["keys"].split()]


def _trees(case, rows):
    """Ancestor masks (bit u: node u is the row's node or an ancestor of it) of one random tree a sequence, parents before children."""
    rng = random.Random(str(rows))
    masks = []
    for n in rows:
        own_masks, depth = [1], [0]
        for v in range(1, n):
            parent = rng.choice([u for u in range(v) if depth[u] < 15][-8:])
            own_masks.append(own_masks[parent] | 1 << v)
            depth.append(depth[parent] + 1)
        masks += own_masks
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device=DEV)


def _normal(gen, *shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device=DEV).normal_(generator=gen)


def _starts(counts):
    return torch.tensor([0] + list(counts), dtype=torch.int64).cumsum(0).to(torch.int32).to(DEV)


def _paged(case, gen, keys):
    """Pages for every sequence's tokens, a few more, in shuffled order; what lies behind a sequence's last token is noise."""
    page = case["page"]
    need = [-(-k // page) for k in keys]
    total = sum(need) + 3
    order = torch.randperm(total, generator=torch.Generator().manual_seed(total)).tolist()
    table = torch.zeros(len(keys), max(need), dtype=torch.int32)
    for s, n in enumerate(need):
        table[s, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    shape = (total, case["kv_heads"], page, case["dim"])
    return _normal(gen, *shape, dtype=TYPES[case["cache"]]), _normal(gen, *shape, dtype=TYPES[case["cache"]]), table.to(DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 13)
    if case["kind"] == "rules":
        return _prepare_rules(case, gen)
    rows, keys = _lengths(case)
    R, dtype = sum(rows), TYPES[case["dtype"]]
    st = {"case": case, "row_start": _starts(rows), "key_len": torch.tensor(keys, dtype=torch.int32, device=DEV), "n_rows": R, "max_rows": max(rows), "max_keys": max(keys),
          "base": None, "mask": None}
    if case["tree"]:
        st["base"] = torch.tensor([k - n for n, k in zip(rows, keys)], dtype=torch.int32, device=DEV)
        st["mask"] = _trees(case, rows)
    q = _normal(gen, R, case["heads"], case["dim"])
    if case["cache"] != "none":
        st["k_cache"], st["v_cache"], st["table"] = _paged(case, gen, keys)
    if case["kind"] == "attend":
        # scores of a few units, and every head's first token drawing some of the weight, as in trained models
        st["q"] = (q * 2.0).to(dtype)
        st["k_cache"][st["table"][:, 0].long(), :, 0] += 0.5 * q[0, :case["kv_heads"]].to(st["k_cache"].dtype)
        h = case["heads"]
        st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, h + 1, device=DEV, dtype=torch.float32) / h) if case["slopes"] else None
        st["prefix"] = torch.tensor([min(case["prefix"], k) for k in keys], dtype=torch.int32, device=DEV) if case["prefix"] else None
        st["out"] = torch.empty_like(st["q"])
        return st
    st["q"] = q.to(dtype)
    st["k"], st["v"] = _normal(gen, R, case["kv_heads"], case["dim"]).to(dtype), _normal(gen, R, case["kv_heads"], case["dim"]).to(dtype)
    st["q_out"] = torch.empty_like(st["q"])
    st["k_out"] = torch.empty_like(st["k"]) if case["cache"] == "none" else None
    st["positions"] = None
    if case["start"] or case["cache"] == "none":
        first = [case["start"] + k - n for n, k in zip(rows, keys)]
        st["positions"] = torch.cat([torch.arange(f, f + n, dtype=torch.int32) for f, n in zip(first, rows)]).to(DEV)
    return st


def _prepare_rules(case, gen):
    S, R, V = case["seqs"], case["seqs"] * case["rows"], case["vocab"]

    def whole(a):
        return torch.tensor(a, dtype=torch.int32, device=DEV)

    def tokens(*shape):
        # a text repeats itself: most of its tokens are from a small part of the vocabulary
        u = torch.rand(*shape, device=DEV, generator=gen)
        return (u ** 3 * V).to(torch.int32).clamp_(0, V - 1)

    lengths = [max(1, case["history"] * (S + i) // (2 * S)) for i in range(S)]
    st = {"case": case, "tokens": tokens(S, max(lengths)), "n_tokens": whole(lengths), "n_prompt": whole([min(case["prompt"], n) for n in lengths]),
          "repetition": 1.0 + 0.3 * torch.rand(S, device=DEV, generator=gen), "presence": 0.5 * torch.rand(S, device=DEV, generator=gen),
          "frequency": 0.3 * torch.rand(S, device=DEV, generator=gen)}
    counts = [max(1, case["bias"] * (i + 1) // S) for i in range(S)]
    st["bias_start"] = _starts(counts)
    st["bias_token"] = torch.cat([torch.randperm(V, generator=gen, device=DEV)[:n] for n in counts]).to(torch.int32)
    st["bias_value"] = _normal(gen, st["bias_token"].numel()) * 4.0
    st["row_start"] = _starts([case["rows"]] * S)
    st["path_token"] = st["path_mask"] = None
    if case["rows"] > 1:
        st["path_token"], st["path_mask"] = tokens(R), _trees(case, [case["rows"]] * S)
    st["allowed"] = st["allowed_row"] = None
    if case["masks"]:
        # a grammar lets a few hundred tokens through at most nodes and nearly all inside free text; some rows have no mask
        words = -(-V // 32)
        bits = torch.rand(R, words * 32, device=DEV, generator=gen) < torch.where(torch.arange(R, device=DEV) % 3 == 0, 0.98, 0.01)[:, None]
        bits[:, V // 2] = True
        st["allowed"] = (bits.view(R, words, 32).long() << torch.arange(32, device=DEV)).sum(-1)
        st["allowed"] = torch.where(st["allowed"] >= 2 ** 31, st["allowed"] - 2 ** 32, st["allowed"]).to(torch.int32)
        st["allowed_row"] = torch.where(torch.arange(R, device=DEV) % 5 == 4, -1, torch.arange(R, device=DEV)).to(torch.int32)
    st["logits"] = (_normal(gen, R, V) * 3.0).to(TYPES[case["dtype"]])
    st["out"] = torch.empty_like(st["logits"])
    return st


# ----------------------------------------------------------------------------- one pass
def run(st):
    return {"rope": _rope, "attend": _attend, "rules": _rules}[st["case"]["kind"]](st)


def _handles(st):
    """What a serving program keeps beside its cache."""
    import paper_2401_15077_amd as pkg
    case, kv = st["case"], None
    if case["cache"] != "none":
        kv = pkg.PagedKV(st["k_cache"], st["v_cache"], st["table"])
    return kv, pkg.Chunk(st["row_start"], st["key_len"], st["n_rows"], st["max_rows"], st["max_keys"], tree_base=st["base"], tree_mask=st["mask"])


def _row_facts(st):
    """Sequence, cache index and position of every row, and its tree bits as truth values [rows, 64] (or None)."""
    r = torch.arange(st["n_rows"], device=DEV)
    start, klen = st["row_start"].long(), st["key_len"].long()
    seq = torch.searchsorted(start, r, right=True) - 1
    index = klen[seq] - start[seq + 1] + r
    if st["mask"] is None:
        return seq, index, index, None
    bits = (st["mask"][:, None] >> torch.arange(64, device=DEV) & 1).bool()
    return seq, index, st["base"].long()[seq] + bits.sum(1) - 1, bits


def _frequencies(case):
    """Radians a position of every pair, in 64 bits."""
    rot, theta, factor = case["rot"], 10000.0, case["factor"]
    p = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    if case["scaling"] == "base":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** (-2.0 * p / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "bands":
        smooth = ((4096.0 * f / (2 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * (smooth + (1.0 - smooth) / factor)
    if case["scaling"] == "ramp":
        def pair(turns):
            return rot * math.log(4096.0 / (2 * math.pi * turns)) / (2 * math.log(theta))
        lo, hi = max(0, math.floor(pair(32.0))), min(rot - 1, math.ceil(pair(1.0)))
        t = ((p - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        f = f * (1.0 - t) + f / factor * t
    return f


def _mscale(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "ramp" else 1.0


def _rope(st):
    case = st["case"]
    if own:
        import paper_2401_15077_amd as pkg
        if "handles" not in st:
            st["handles"] = _handles(st)
            st["plan"] = pkg.rope_plan(case["dim"], theta=10000.0, rot_dim=case["rot"], interleaved=case["layout"] == "pairs", scaling=case["scaling"], factor=case["factor"],
                                       low=1.0, high=32.0 if case["scaling"] == "ramp" else 4.0, trained_len=4096, mscale=_mscale(case))
        kv, chunk = st["handles"]
        if kv is None:
            pkg.rope(st["plan"], st["q"], st["k"], positions=st["positions"], q_out=st["q_out"], k_out=st["k_out"], inverse=case["inverse"])
            return {"q": st["q_out"], "k": st["k_out"]}
        pkg.rope(st["plan"], st["q"], st["k"], st["v"], chunk=chunk, kv=kv, positions=st["positions"], q_out=st["q_out"], inverse=case["inverse"])
        return {"q": st["q_out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    seq, index, position, _ = _row_facts(st)
    if st["positions"] is not None:
        position = st["positions"]
    angle = position.double()[:, None] * _frequencies(case)
    if case["inverse"]:
        angle = -angle
    m = _mscale(case)
    cos, sin = (angle.cos() * m).float()[:, None], (angle.sin() * m).float()[:, None]
    rot = case["rot"]

    def rotate(x):
        x = x.float()
        y = x.clone()
        a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y

    q, k = rotate(st["q"]).to(st["q"].dtype), rotate(st["k"])
    if case["cache"] == "none":
        return {"q": q, "k": k.to(st["k"].dtype)}
    where = st["table"].long()[seq, index // case["page"]], slice(None), index % case["page"]
    st["k_cache"][where] = k.to(st["k_cache"].dtype)
    st["v_cache"][where] = st["v"].to(st["v_cache"].dtype)
    return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _attend(st):
    case = st["case"]
    if own:
        import paper_2401_15077_amd as pkg
        if "handles" not in st:
            st["handles"] = _handles(st)
            st["workspace"] = torch.empty(pkg.chunk_attention_workspace(st["q"], *st["handles"]), dtype=torch.uint8, device=DEV)
        kv, chunk = st["handles"]
        return pkg.chunk_attention(st["q"], kv, chunk, softcap=case["softcap"], slopes=st["slopes"], window=case["window"], prefix=st["prefix"], out=st["out"],
                                   workspace=st["workspace"])
    H, KVH, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    seq, index, position, bits = _row_facts(st)
    S, g, n, K = st["key_len"].numel(), H // KVH, st["max_rows"], st["max_keys"]
    # rows and tokens of all sequences side by side, padded
    start, count = st["row_start"].long()[:-1], st["row_start"].long().diff()
    i = torch.arange(n, device=DEV)
    row = (start[:, None] + i).clamp(max=st["n_rows"] - 1)                         # [S, n]
    j = torch.arange(K, device=DEV)
    pages = st["table"].long()[:, :-(-K // page)]
    k = st["k_cache"][pages].transpose(1, 2).reshape(S, KVH, -1, dim)[:, :, :K].float()
    v = st["v_cache"][pages].transpose(1, 2).reshape(S, KVH, -1, dim)[:, :, :K].float()
    own_index, own_position = index[row][:, :, None], position[row][:, :, None]
    if bits is None:
        ordered, key_position = j <= own_index, j[None, None]
    else:
        past = j - st["base"].long()[:, None]                                       # [S, K]: index among the tree's nodes
        node = past.clamp(0, 63)[:, None].expand(S, n, K)
        mine = bits[row]                                                            # [S, n, 64]
        ordered = (past[:, None] < 0) | (mine.gather(2, node) & (past < 64)[:, None])
        before = mine.long().cumsum(2) - mine.long()                                # ancestors in front of a node
        key_position = torch.where(past[:, None] < 0, j[None, None], st["base"].long()[:, None, None] + before.gather(2, node))
    distance = own_position - key_position
    seen = ordered & (distance < case["window"]) if case["window"] else ordered
    if st["prefix"] is not None:
        prefix = st["prefix"].long() if bits is None else torch.minimum(st["prefix"].long(), st["base"].long())
        seen = seen | (j < prefix[:, None])[:, None]
    seen = seen & (j < st["key_len"].long()[:, None])[:, None] & (i < count[:, None])[:, :, None]
    q = st["q"].float()[row].view(S, n, KVH, g, dim).permute(0, 2, 3, 1, 4).reshape(S, KVH, g * n, dim)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).view(S, KVH, g, n, K) * dim ** -0.5
    if case["softcap"]:
        score = case["softcap"] * torch.tanh(score / case["softcap"])
    if case["slopes"]:
        score = score - st["slopes"].view(KVH, g, 1, 1) * distance.abs().float()[:, None, None]
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul((weight / torch.where(total > 0, total, 1.0)).view(S, KVH, g * n, K), v)
    out = out.view(S, H, n, dim).transpose(1, 2)                                    # [S, n, H, dim]
    return out[seq, torch.arange(st["n_rows"], device=DEV) - start[seq]].to(st["q"].dtype)


def _rules(st):
    case = st["case"]
    if own:
        import paper_2401_15077_amd as pkg
        if "handles" not in st:
            st["handles"] = pkg.LogitRules(st["tokens"], st["n_tokens"], n_prompt=st["n_prompt"], repetition=st["repetition"], presence=st["presence"],
                                           frequency=st["frequency"], bias=(st["bias_start"], st["bias_token"], st["bias_value"]))
        return pkg.apply_logit_rules(st["logits"], st["handles"], row_start=st["row_start"], path_token=st["path_token"], path_mask=st["path_mask"],
                                     allowed=st["allowed"], allowed_row=st["allowed_row"], out=st["out"])
    S, R, V, L = case["seqs"], st["logits"].shape[0], case["vocab"], st["tokens"].shape[1]
    seq = torch.arange(R, device=DEV) // case["rows"]
    at = torch.arange(L, device=DEV)
    there = at < st["n_tokens"].long()[:, None]
    new = there & (at >= st["n_prompt"].long()[:, None])
    seen = torch.zeros(S, V, device=DEV).scatter_add_(1, st["tokens"].long(), there.float())[seq]
    count = torch.zeros(S, V, device=DEV).scatter_add_(1, st["tokens"].long(), new.float())[seq]
    if st["path_mask"] is not None:
        bits = (st["path_mask"][:, None] >> torch.arange(case["rows"], device=DEV) & 1).float()
        path = st["path_token"].view(S, -1).long()[seq]                             # [R, nodes]
        seen = seen.scatter_add(1, path, bits)
        count = count.scatter_add(1, path, bits)
    x = st["logits"].float()
    rep = st["repetition"][seq][:, None]
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - torch.where(count > 0, st["presence"][seq][:, None] + st["frequency"][seq][:, None] * count, 0.0)
    of = torch.searchsorted(st["bias_start"].long(), torch.arange(st["bias_token"].numel(), device=DEV), right=True) - 1
    bias = torch.zeros(S, V, device=DEV)
    bias[of, st["bias_token"].long()] = st["bias_value"]
    x = x + bias[seq]
    if st["allowed"] is not None:
        words = st["allowed"][st["allowed_row"].long().clamp(min=0)]
        ok = (words[:, :, None] >> torch.arange(32, device=DEV) & 1).bool().view(R, -1)[:, :V]
        x = x.masked_fill(~ok & (st["allowed_row"] >= 0)[:, None], -math.inf)
    return x.to(st["logits"].dtype)


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "rules":
        S, R, V, elt = case["seqs"], case["seqs"] * case["rows"], case["vocab"], 4 if case["dtype"] == "fp32" else 2
        lists = sum(max(1, case["history"] * (S + i) // (2 * S)) for i in range(S)) * 4 + sum(max(1, case["bias"] * (i + 1) // S) for i in range(S)) * 8
        masks = sum(i % 5 != 4 for i in range(R)) * V / 8 if case["masks"] else 0
        return {"bytes": 2.0 * R * V * elt + lists + masks + (12 * R if case["rows"] > 1 else 0), "flops": 5.0 * R * V}
    rows, keys = _lengths(case)
    H, KVH, dim, R = case["heads"], case["kv_heads"], case["dim"], sum(rows)
    elt, kv_elt = 4 if case["dtype"] == "fp32" else 2, 4 if case["cache"] == "fp32" else 2
    if case["kind"] == "rope":
        rotated = 6.0 * R * (H + KVH) * case["rot"] / 2
        if case["cache"] == "none":
            return {"bytes": 2.0 * R * (H + KVH) * dim * elt, "flops": rotated}
        return {"bytes": float(R * dim * (2 * H * elt + 2 * KVH * (elt + kv_elt))), "flops": rotated}
    pairs = read = 0
    masks = _tree_bits(case, rows)
    for s, (n, K) in enumerate(zip(rows, keys)):
        base = K - n
        window = case["window"] or 1 << 30
        first = K                                    # keys that some row sees, apart from the prefix
        for i in range(n):
            own_position = base + (bin(masks[s][i]).count("1") - 1 if case["tree"] else i)
            lo = max(0, own_position - window + 1)   # first visible token by distance, if it lies in front of the chunk
            prefix = min(case["prefix"], base if case["tree"] else K)
            if case["tree"]:
                visible = max(0, base - lo) + min(own_position - base + 1, window)
            else:
                visible = own_position + 1 - lo
            pairs += visible + (min(prefix, lo) if case["tree"] else min(prefix, lo) + max(0, prefix - own_position - 1))
            first = min(first, lo)
        read += K - first + min(case["prefix"], first)
    return {"bytes": 2.0 * R * H * dim * elt + 2.0 * read * KVH * dim * kv_elt, "flops": 4.0 * dim * H * pairs}


def _tree_bits(case, rows):
    if not case["tree"]:
        return None
    flat = [m % (1 << 64) for m in _trees(case, rows).tolist()]
    return [[flat.pop(0) for _ in range(n)] for n in rows]


# ----------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "rules": _exact_rules}[case["kind"]](case, st)


def _ancestors(masks, s, i):
    return [u for u in range(64) if masks[s][i] >> u & 1]


def _exact_rope(case, st):
    rows, keys = _lengths(case)
    masks = _tree_bits(case, rows)
    rot, factor, L = case["rot"], case["factor"], 4096
    turns = []                                        # radians a position, pair by pair
    for p in range(rot // 2):
        f = math.exp(-2.0 * p / rot * math.log(10000.0))
        if case["scaling"] == "linear":
            f /= factor
        elif case["scaling"] == "base":
            f = math.exp(-2.0 * p / rot * (math.log(10000.0) + rot / (rot - 2) * math.log(factor)))
        elif case["scaling"] == "bands":
            wave = 2 * math.pi / f
            if wave > L / 1.0:
                f /= factor
            elif wave >= L / 4.0:
                s = (L / wave - 1.0) / (4.0 - 1.0)
                f = (1 - s) * f / factor + s * f
        elif case["scaling"] == "ramp":
            lo = max(math.floor(rot * math.log(L / (32.0 * 2 * math.pi)) / (2 * math.log(10000.0))), 0)
            hi = min(math.ceil(rot * math.log(L / (1.0 * 2 * math.pi)) / (2 * math.log(10000.0))), rot - 1)
            t = min(1.0, max(0.0, (p - lo) / max(hi - lo, 0.001)))
            f = f / factor * t + f * (1 - t)
        turns.append(f)
    indices, positions = [], []
    for s, (n, K) in enumerate(zip(rows, keys)):
        for i in range(n):
            indices.append((s, K - n + i))
            positions.append(K - n + (len(_ancestors(masks, s, i)) - 1 if masks else i) + case["start"])
    phase = torch.tensor(positions, dtype=torch.float64, device=DEV)[:, None] * torch.tensor(turns, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(phase, _mscale(case)), -phase if case["inverse"] else phase)[:, None]

    def rotated(x):
        x = x.double()
        head, rest = x[..., :rot], x[..., rot:]
        if case["layout"] == "half":
            z = torch.complex(head[..., :rot // 2], head[..., rot // 2:]) * turn
            return torch.cat([z.real, z.imag, rest], -1)
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous()) * turn
        return torch.cat([torch.view_as_real(z).flatten(-2), rest], -1)

    if case["cache"] == "none":
        return {"q": rotated(st["q"]), "k": rotated(st["k"])}
    k_cache, v_cache = st["k_cache"].double(), st["v_cache"].double()
    table = st["table"].tolist()
    page = torch.tensor([table[s][i // case["page"]] for s, i in indices], device=DEV)
    slot = torch.tensor([i % case["page"] for _, i in indices], device=DEV)
    k_cache[page, :, slot], v_cache[page, :, slot] = rotated(st["k"]), st["v"].double()
    return {"q": rotated(st["q"]), "k_cache": k_cache, "v_cache": v_cache}


def _exact_attend(case, st):
    rows, keys = _lengths(case)
    masks = _tree_bits(case, rows)
    H, KVH, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    g, at = H // KVH, 0
    out = torch.zeros(sum(rows), H, dim, dtype=torch.float64, device=DEV)
    for s, (n, K) in enumerate(zip(rows, keys)):
        base, slot = K - n, torch.arange(K, device=DEV)
        cells = st["table"][s].long()[slot // page], slice(None), slot % page
        k, v = st["k_cache"][cells].double(), st["v_cache"][cells].double()            # [K, KVH, dim]
        if case["tree"]:
            far = torch.empty(n, K, dtype=torch.float64)
            far[:] = math.nan                                                          # (nan: not on the row's path)
            for i in range(n):
                path = _ancestors(masks, s, i)
                far[i, :base] = base + len(path) - 1 - torch.arange(base)
                far[i, [base + u for u in path]] = torch.arange(len(path) - 1, -1, -1).double()
            far = far.to(DEV)
            seen = ~far.isnan()
            far = far.nan_to_num(0.0)
        else:
            far = (base + torch.arange(n, device=DEV, dtype=torch.float64))[:, None] - slot
            seen = far >= 0
        if case["window"]:
            seen = seen & (far < case["window"])
        if case["prefix"]:
            seen[:, :min(case["prefix"], base if case["tree"] else K)] = True
        for h in range(H):
            z = st["q"][at:at + n, h].double() @ k[:, h // g].T / math.sqrt(dim)
            if case["softcap"]:
                z = torch.tanh(z / case["softcap"]) * case["softcap"]
            if case["slopes"]:
                z = z - float(st["slopes"][h]) * far.abs()
            out[at:at + n, h] = torch.softmax(z.masked_fill(~seen, -math.inf), -1) @ v[:, h // g]
        at += n
    return out


def _exact_rules(case, st):
    S, rows, V = case["seqs"], case["rows"], case["vocab"]
    masks = None if st["path_mask"] is None else [m % (1 << 64) for m in st["path_mask"].tolist()]
    out = st["logits"].double()
    for s in range(S):
        n, prompt = int(st["n_tokens"][s]), int(st["n_prompt"][s])
        text = st["tokens"][s, :n].long()
        said, fresh = torch.bincount(text, minlength=V), torch.bincount(text[prompt:], minlength=V)
        b0, b1 = int(st["bias_start"][s]), int(st["bias_start"][s + 1])
        rep, pres, freq = (float(st[name][s]) for name in ("repetition", "presence", "frequency"))
        for r in range(s * rows, (s + 1) * rows):
            path = torch.zeros(0, dtype=torch.int64, device=DEV)
            if masks is not None:
                path = st["path_token"][torch.tensor([s * rows + u for u in range(rows) if masks[r] >> u & 1], device=DEV)].long()
            more = torch.bincount(path, minlength=V)
            x, c = out[r], fresh + more
            x = torch.where(said + more > 0, torch.where(x > 0, x / rep, x * rep), x)
            x = x - (c > 0) * pres - freq * c
            x[st["bias_token"][b0:b1].long()] += st["bias_value"][b0:b1].double()
            if st["allowed"] is not None and int(st["allowed_row"][r]) >= 0:
                word = st["allowed"][int(st["allowed_row"][r])]
                t = torch.arange(V, device=DEV)
                x[(word[t // 32] >> (t % 32) & 1) == 0] = -math.inf
            out[r] = x
    return out
