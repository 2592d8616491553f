"""Timed cases of the operators around a cache held in 8 bits, and of the choice of a token: the append of keys and values (rotated on the way) to a paged cache of 8-bit
codes with a scale for each block of tokens and head, attention of a chunk of new tokens over it, and sampling with temperature, top-k, top-p and min-p from given random numbers.

Every case is a call that a serving program makes with the tensors it has in hand.  `own` chooses between the plain form (elementary torch operations in 32 bits; angles, codes and masses in 64)
and the library's operators; `exact` is the definition in 64 bits.  Lengths, trees and page tables are functions of the case, values of the seed.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
LARGEST = {"e4m3": 448.0, "int8": 127.0}


def listed():
    def append(name, rows, keys, heads, kv_heads, dim, dtype, cache, block, tree=False, layout="half", rot=0, start=0, page=64):
        return {"name": name, "kind": "append", "rows": rows, "keys": keys, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache, "block": block,
                "tree": tree, "layout": layout, "rot": rot or dim, "start": start, "page": page}

    def attend(name, rows, keys, heads, kv_heads, dim, dtype, cache, block, tree=False, softcap=0.0, window=0, slopes=False, prefix=0, page=64):
        return {"name": name, "kind": "attend", "rows": rows, "keys": keys, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache, "block": block,
                "tree": tree, "softcap": softcap, "window": window, "slopes": slopes, "prefix": prefix, "page": page}

    def sample(name, rows, vocab, dtype, filters, masks=False):
        return {"name": name, "kind": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "filters": filters, "masks": masks}

    batch = " ".join(str(1024 + 241 * i) for i in range(64))
    # rows and keys: one number a sequence, new tokens and tokens in the cache with them
    return [
        # one user, one new token that joins 12 others in its block: nothing but latency
        append("append8-token", "1", "701", 32, 32, 128, "fp32", "e4m3", 16),
        # four users' draft trees behind their texts; half of a head rotated in adjacent pairs; a scale a page
        append("append8-trees", "26 26 26 26", "1526 2051 1787 2330", 32, 8, 128, "fp32", "int8", 64, tree=True, layout="pairs", rot=64),
        # a full serving batch, one token each
        append("append8-batch", "1 " * 64, batch, 64, 8, 128, "bf16", "e4m3", 16),
        # chunks of five long prompts on the way into the cache, far into a document
        append("append8-chunks", "4096 2011 1 1500 583", "4096 2100 777 1500 1024", 64, 8, 128, "bf16", "e4m3", 32, start=90000),
        # one user, one new token, fp32 rows
        attend("attend8-token", "1", "701", 32, 32, 128, "fp32", "e4m3", 16),
        # four users' draft trees: 104 rows
        attend("attend8-trees", "26 26 26 26", "1526 2051 1787 2330", 32, 8, 128, "fp32", "int8", 64, tree=True),
        # a full serving batch, one token each, contexts of a thousand to sixteen thousand tokens
        attend("attend8-batch", "1 " * 64, batch, 64, 8, 128, "bf16", "e4m3", 64),
        # chunks of two prompts in the middle of a document: capped scores, a sliding window
        attend("attend8-chunks", "1536 509", "7536 2509", 32, 8, 128, "bf16", "e4m3", 32, softcap=50.0, window=4096),
        # one user, one token, every filter
        sample("sample-token", 1, 32000, "fp32", "all"),
        # four users' draft trees under a grammar, each row with filters of its own
        sample("sample-trees", 104, 32000, "fp32", "mixed", True),
        # a few users of a large vocabulary who set a temperature only
        sample("sample-few", 3, 128256, "fp32", "none"),
        # a serving batch, half-width logits of a large odd vocabulary, nucleus sampling
        sample("sample-batch", 160, 100003, "bf16", "nucleus"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "sample"])
    if kind == "sample":
        return {"kind": "sample", "rows": _log_int(rng, 1, 150), "vocab": _log_int(rng, 900, 100003), "dtype": rng.choice(["fp32", "bf16"]),
                "filters": rng.choice(["all", "mixed", "nucleus", "top", "least", "none"]), "masks": rng.random() < 0.3}
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (64, 8), (40, 40), (8, 2), (12, 4), (5, 1)])
    dim = rng.choice([128, 128, 128, 64, 80, 32])
    dtype = rng.choice(["fp32", "bf16"])
    cache = rng.choice(["e4m3", "int8"])
    page = rng.choice([16, 32, 64, 128])
    block = rng.choice([b for b in (16, 32, 64, 128) if b <= page])
    tree = rng.random() < 0.3
    if kind == "append":
        shape = "tree" if tree else rng.choice(["token", "chunk"])
        seqs = _log_int(rng, 1, 48) if shape == "token" else rng.randint(1, 6)
        rows = [{"tree": rng.randint(2, 64), "token": rng.choice([1, 1, 1, 2, 7]), "chunk": _log_int(rng, 1, 1200)}[shape] for _ in range(seqs)]
        keys = [n + (0 if rng.random() < 0.2 else _log_int(rng, 1, 2000)) for n in rows]
        return {"kind": "append", "rows": " ".join(map(str, rows)), "keys": " ".join(map(str, keys)), "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache,
                "block": block, "tree": tree, "layout": rng.choice(["half", "pairs"]), "rot": rng.choice([dim, dim, dim // 2]),
                "start": 0 if tree or rng.random() < 0.5 else _log_int(rng, 1, 30000), "page": page}
    shape = "tree" if tree else rng.choice(["token", "token", "chunk"])
    seqs = {"tree": rng.randint(1, 6), "token": _log_int(rng, 1, 32), "chunk": rng.randint(1, 3)}[shape]
    rows = [{"tree": rng.randint(2, 64), "token": rng.choice([1, 1, 1, 2, 7]), "chunk": _log_int(rng, 20, 1000)}[shape] for _ in range(seqs)]
    keys = [n + (0 if rng.random() < 0.1 else _log_int(rng, 1, {"tree": 3000, "token": 6000, "chunk": 2500}[shape])) for n in rows]
    return {"kind": "attend", "rows": " ".join(map(str, rows)), "keys": " ".join(map(str, keys)), "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache,
            "block": block, "tree": tree, "softcap": rng.choice([0.0, 0.0, 30.0]), "window": rng.choice([0, 0, _log_int(rng, 16, 2000)]), "slopes": rng.random() < 0.3,
            "prefix": rng.choice([0, 0, _log_int(rng, 1, 500)]), "page": page}


# ----------------------------------------------------------------------------- inputs
def _lengths(case):
    return [int(x) for x in case["rows"].split()], [int(x) for x in case["keys"].split()]


def _trees(rows):
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


def _normal(gen, *shape):
    return torch.empty(*shape, dtype=torch.float32, device=DEV).normal_(generator=gen)


def _starts(counts):
    return torch.tensor([0] + list(counts), dtype=torch.int64).cumsum(0).to(torch.int32).to(DEV)


def _held(x, cache, block, whole_powers):
    """Codes and scales of x [pages, heads, tokens, dim]: scales as an append leaves them (powers of two), or as a calibration does (the largest code stands for the largest value)."""
    P, H, N, D = x.shape
    x = x.view(P, H, N // block, block * D)
    scale = x.abs().amax(-1) / LARGEST[cache]
    if whole_powers:
        scale = torch.exp2(torch.ceil(torch.log2(scale)))
    x = x / scale[..., None]
    codes = x.to(CODES[cache]) if cache == "e4m3" else x.round().to(torch.int8)
    return codes.view(P, H, N, D), scale


def _paged(case, gen, keys):
    """Pages for every sequence's tokens, a few more, in shuffled order; what lies behind a sequence's last token is as large as the rest."""
    page, whole = case["page"], case["kind"] == "append"
    need = [-(-k // page) for k in keys]
    total = sum(need) + 3
    order = torch.randperm(total, generator=torch.Generator().manual_seed(total)).tolist()
    table = torch.zeros(len(keys), max(need), dtype=torch.int32)
    for s, n in enumerate(need):
        table[s, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    shape = (total, case["kv_heads"], page, case["dim"])
    table = table.to(DEV)
    k = _normal(gen, *shape)
    if not whole:
        # every head's first token draws some of the weight, as in trained models
        k[table[:, 0].long(), :, 0] += 0.5 * _normal(gen, case["kv_heads"], case["dim"])
    k = _held(k, case["cache"], case["block"], whole)
    return k, _held(_normal(gen, *shape), case["cache"], case["block"], whole), table


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 29)
    if case["kind"] == "sample":
        return _prepare_sample(case, gen)
    rows, keys = _lengths(case)
    R, dtype = sum(rows), TYPES[case["dtype"]]
    st = {"case": case, "row_start": _starts(rows), "key_len": torch.tensor(keys, dtype=torch.int32, device=DEV), "n_rows": R, "max_rows": max(rows), "max_keys": max(keys),
          "base": None, "mask": None}
    if case["tree"]:
        st["base"] = torch.tensor([k - n for n, k in zip(rows, keys)], dtype=torch.int32, device=DEV)
        st["mask"] = _trees(rows)
    q = _normal(gen, R, case["heads"], case["dim"])
    (st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"]), st["table"] = _paged(case, gen, keys)
    if case["kind"] == "attend":
        st["q"] = (q * 2.0).to(dtype)                    # scores of a few units
        h = case["heads"]
        st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, h + 1, device=DEV, dtype=torch.float32) / h) if case["slopes"] else None
        st["prefix"] = torch.tensor([min(case["prefix"], k) for k in keys], dtype=torch.int32, device=DEV) if case["prefix"] else None
        st["out"] = torch.empty_like(st["q"])
        return st
    st["q"] = q.to(dtype)
    # some tokens are larger than what their block was scaled for
    st["k"], st["v"] = ((_normal(gen, R, case["kv_heads"], case["dim"]) * torch.exp(0.4 * _normal(gen, R, 1, 1))).to(dtype) for _ in range(2))
    st["q_out"] = torch.empty_like(st["q"])
    st["positions"] = None
    if case["start"]:
        first = [case["start"] + k - n for n, k in zip(rows, keys)]
        st["positions"] = torch.cat([torch.arange(f, f + n, dtype=torch.int32) for f, n in zip(first, rows)]).to(DEV)
    return st


def _prepare_sample(case, gen):
    R, V, filters = case["rows"], case["vocab"], case["filters"]
    # a few tokens stand out, more in some rows than in others
    x = _normal(gen, R, V) * (1.5 + 2.0 * torch.rand(R, 1, device=DEV, generator=gen))
    x += (torch.rand(R, V, device=DEV, generator=gen) < 20.0 / V).float() * 8.0 * torch.rand(R, 1, device=DEV, generator=gen)
    if case["masks"]:
        # a grammar has left a few hundred tokens at most nodes and nearly all inside free text
        kept = torch.rand(R, V, device=DEV, generator=gen) < torch.where(torch.arange(R, device=DEV) % 3 == 0, 0.98, min(1.0, 300.0 / V))[:, None]
        kept[:, V // 2] = True
        x = x.masked_fill(~kept, -math.inf)
    r = torch.arange(R, device=DEV)
    st = {"case": case, "logits": x.to(TYPES[case["dtype"]]), "uniform": torch.rand(R, device=DEV, generator=gen), "temperature": 0.6 + 0.6 * torch.rand(R, device=DEV, generator=gen),
          "top_k": None, "top_p": None, "min_p": None, "token": torch.empty(R, dtype=torch.int32, device=DEV), "logprob": torch.empty(R, device=DEV)}
    k, p, m = torch.randint(20, 100, (R,), device=DEV, generator=gen, dtype=torch.int32), 0.8 + 0.19 * torch.rand(R, device=DEV, generator=gen), 0.02 + 0.1 * torch.rand(R, device=DEV, generator=gen)
    if filters == "mixed":
        st["temperature"] = torch.where(r % 9 == 8, 0.0, st["temperature"])
        st["top_k"], st["top_p"], st["min_p"] = torch.where(r % 4 < 2, k, 0), torch.where(r % 2 == 0, p, 1.0), torch.where(r % 4 == 3, m, 0.0)
    if filters in ("all", "top"):
        st["top_k"] = k
    if filters in ("all", "nucleus"):
        st["top_p"] = p
    if filters in ("all", "least"):
        st["min_p"] = m
    return st


# ----------------------------------------------------------------------------- one pass
def run(st):
    return {"append": _append, "attend": _attend, "sample": _sample}[st["case"]["kind"]](st)


def _handles(st):
    """What a serving program keeps beside its cache."""
    import paper_2401_15077_amd as pkg
    return (pkg.PagedKV8(st["k_cache"], st["v_cache"], st["table"], st["k_scale"], st["v_scale"]),
            pkg.Chunk(st["row_start"], st["key_len"], st["n_rows"], st["max_rows"], st["max_keys"], tree_base=st["base"], tree_mask=st["mask"]))


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


def _exponent(a, largest):
    """The least whole e with a <= largest * 2^e."""
    e = torch.ceil(torch.log2(a / largest))
    e = torch.where(a <= largest * torch.exp2(e - 1), e - 1, e)
    return torch.where(a > largest * torch.exp2(e), e + 1, e)


def _rounded(x, cache):
    """Codes of x (64 bits), as numbers: to nearest, ties to even, within the largest code."""
    if cache == "int8":
        return x.round().clamp(-127.0, 127.0)
    step = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=-6).double() - 3.0)
    return ((x / step).round() * step).clamp(-448.0, 448.0)


def _append(st):
    case = st["case"]
    outputs = {"q": st["q_out"], "k": st["k_cache"], "v": st["v_cache"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}
    if own:
        import paper_2401_15077_amd as pkg
        if "handles" not in st:
            st["handles"] = _handles(st)
            st["plan"] = pkg.rope_plan(case["dim"], theta=10000.0, rot_dim=case["rot"], interleaved=case["layout"] == "pairs")
        kv, chunk = st["handles"]
        pkg.rope(st["plan"], st["q"], st["k"], st["v"], chunk=chunk, kv=kv, positions=st["positions"], q_out=st["q_out"])
        return outputs
    seq, index, position, _ = _row_facts(st)
    if st["positions"] is not None:
        position = st["positions"]
    rot, page, B = case["rot"], case["page"], case["block"]
    p = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    angle = position.double()[:, None] * 10000.0 ** (-2.0 * p / rot)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def rotate(x, cos, sin):
        y = x.clone()
        a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y

    st["q_out"].copy_(rotate(st["q"].float(), cos.float(), sin.float()))
    # the blocks that the rows go to: page, first slot, the sequence's tokens in it, those that are written now
    per_page = page // B
    name, of = torch.unique(st["table"].long()[seq, index // page] * per_page + index % page // B, return_inverse=True)
    n = name.numel()
    first = torch.empty(n, dtype=torch.int64, device=DEV)
    last = torch.empty_like(first)
    first[of], last[of] = index // B * B, st["key_len"].long()[seq]
    slot = torch.arange(B, device=DEV)
    written = torch.zeros(n, B, dtype=torch.bool, device=DEV)
    written[of, index % B] = True
    other = (first[:, None] + slot < last[:, None]) & ~written                       # tokens that stay
    cell = (name // per_page)[:, None].expand(n, B), (name % per_page * B)[:, None] + slot

    def put(x, codes, scale):
        """x: rows in 64 bits."""
        largest = LARGEST[case["cache"]]
        a = torch.zeros(n, x.shape[1], dtype=torch.float64, device=DEV)
        a.scatter_reduce_(0, of[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
        old_scale = scale[name // per_page, :, name % per_page].double()
        grown = _exponent(a / old_scale, largest).clamp(min=0.0)
        new_scale = torch.where(other.any(1)[:, None], old_scale * torch.exp2(grown), torch.exp2(_exponent(a, largest).clamp(-100.0, 100.0)))
        scale[name // per_page, :, name % per_page] = new_scale.float()
        held = codes.view(torch.uint8).transpose(1, 2)[cell].view(codes.dtype).double()   # [blocks, B, heads, dim]
        held = torch.where(other[:, :, None, None], _rounded(held * torch.exp2(-grown)[:, None, :, None], case["cache"]), held)
        held[of, index % B] = _rounded(x / new_scale[of][:, :, None], case["cache"])
        codes.view(torch.uint8).transpose(1, 2)[cell] = held.float().to(codes.dtype).view(torch.uint8)

    put(rotate(st["k"].double(), cos, sin), st["k_cache"], st["k_scale"])
    put(st["v"].double(), st["v_cache"], st["v_scale"])
    return outputs


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

    def values(codes, scale):
        x = codes.view(torch.uint8)[pages].view(codes.dtype).float()                # [S, pages, heads, tokens, dim]
        x = x.view(*x.shape[:3], -1, case["block"], dim) * scale[pages][..., None, None]
        return x.view(S, -1, KVH, page, dim).transpose(1, 2).reshape(S, KVH, -1, dim)[:, :, :K]

    k, v = values(st["k_cache"], st["k_scale"]), values(st["v_cache"], st["v_scale"])
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


def _sample(st):
    if own:
        import paper_2401_15077_amd as pkg
        if "workspace" not in st:
            st["workspace"] = torch.empty(pkg.sample_workspace(st["logits"]), dtype=torch.uint8, device=DEV)
        pkg.sample(st["logits"], st["uniform"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"], token=st["token"], logprob=st["logprob"],
                   workspace=st["workspace"])
        return {"token": st["token"], "logprob": st["logprob"]}
    x, order = torch.sort(st["logits"].double(), dim=1, descending=True, stable=True)
    greedy = st["temperature"] <= 0
    t = (x - x[:, :1]) / torch.where(greedy, 1.0, st["temperature"]).double()[:, None]
    mass, rank = torch.exp(t), torch.arange(x.shape[1], device=DEV)
    kept = (rank == 0) | ~greedy[:, None]
    if st["top_k"] is not None:
        kept = kept & ((rank < st["top_k"][:, None]) | (st["top_k"] <= 0)[:, None])
    if st["top_p"] is not None:
        m = torch.where(kept, mass, 0.0)
        sums = m.cumsum(1)
        kept = kept & ((sums - m < st["top_p"].double()[:, None] * sums[:, -1:]) | (st["top_p"] >= 1)[:, None] | (rank == 0))
    if st["min_p"] is not None:
        kept = kept & ((t >= torch.log(st["min_p"].double())[:, None]) | (rank == 0))
    mass = torch.where(kept, mass, 0.0)
    sums = mass.cumsum(1)
    at = torch.minimum((sums <= st["uniform"].double()[:, None] * sums[:, -1:]).sum(1), kept.sum(1) - 1)[:, None]
    return {"token": order.gather(1, at)[:, 0].to(torch.int32), "logprob": torch.log(mass.gather(1, at) / sums[:, -1:])[:, 0].float()}


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "sample":
        R, V = case["rows"], case["vocab"]
        return {"bytes": float(R * V * (4 if case["dtype"] == "fp32" else 2) + 24 * R), "flops": 3.0 * R * V}
    rows, keys = _lengths(case)
    H, KVH, dim, R, block = case["heads"], case["kv_heads"], case["dim"], sum(rows), case["block"]
    elt = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "append":
        blocks = sum((k - 1) // block - (k - n) // block + 1 for n, k in zip(rows, keys))
        return {"bytes": float(R * dim * (2 * H * elt + 2 * KVH * (elt + 1)) + 16 * blocks * KVH), "flops": 6.0 * R * (H + KVH) * case["rot"] / 2 + 4.0 * R * KVH * dim}
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
    return {"bytes": 2.0 * R * H * dim * elt + 2.0 * read * KVH * (dim + 4 / block), "flops": 4.0 * dim * H * pairs}


def _tree_bits(case, rows):
    if not case["tree"]:
        return None
    flat = [m % (1 << 64) for m in _trees(rows).tolist()]
    return [[flat.pop(0) for _ in range(n)] for n in rows]


# ----------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["kind"]](case, st)


def _ancestors(masks, s, i):
    return [u for u in range(64) if masks[s][i] >> u & 1]


def _nearest(x, cache):
    """Codes of the numbers x (numpy, 64 bits)."""
    if cache == "int8":
        return np.clip(np.rint(x), -127, 127)
    size = np.maximum(np.abs(x), 2.0 ** -6)
    unit = 2.0 ** (np.floor(np.log2(size)) - 3)
    unit = np.where(size >= 16 * unit, 2 * unit, np.where(size < 8 * unit, unit / 2, unit))
    return np.clip(np.rint(x / unit) * unit, -448.0, 448.0)


def _exact_append(case, st):
    rows, keys = _lengths(case)
    masks = _tree_bits(case, rows)
    rot, page, B, cache = case["rot"], case["page"], case["block"], case["cache"]
    positions = [case["start"] + K - n + (len(_ancestors(masks, s, i)) - 1 if masks else i) for s, (n, K) in enumerate(zip(rows, keys)) for i in range(n)]
    turns = [math.exp(-2.0 * p / rot * math.log(10000.0)) for p in range(rot // 2)]
    phase = np.array(positions, dtype=np.float64)[:, None] * np.array(turns)
    turn = (np.cos(phase) + 1j * np.sin(phase))[:, None]

    def rotated(x):
        x = x.double().cpu().numpy().copy()
        if case["layout"] == "half":
            z = (x[..., :rot // 2] + 1j * x[..., rot // 2:rot]) * turn
            x[..., :rot // 2], x[..., rot // 2:rot] = z.real, z.imag
        else:
            z = (x[..., :rot:2] + 1j * x[..., 1:rot:2]) * turn
            x[..., :rot:2], x[..., 1:rot:2] = z.real, z.imag
        return x

    table = st["table"].tolist()

    def stored(x, codes, scale):
        codes, scale = codes.float().double().cpu().numpy(), scale.double().cpu().numpy()
        at = 0
        for s, (n, K) in enumerate(zip(rows, keys)):
            for b in range((K - n) // B, (K - 1) // B + 1):
                lo, hi = max(K - n, b * B), min(K, b * B + B)                    # tokens that are written
                new = x[at + lo - (K - n):at + hi - (K - n)]                     # [tokens, heads, dim]
                p, slot = table[s][b * B // page], b * B % page
                size = np.abs(new).max(axis=(0, 2))
                for h, a in enumerate(size):
                    old = lo > b * B
                    unit = scale[p, h, slot // B] if old else 2.0 ** -100
                    while a > LARGEST[cache] * unit:
                        unit *= 2.0
                    if old and unit > scale[p, h, slot // B]:
                        stay = codes[p, h, slot:slot + lo - b * B]
                        stay[:] = _nearest(stay * (scale[p, h, slot // B] / unit), cache)
                    scale[p, h, slot // B] = unit
                    codes[p, h, slot + lo - b * B:slot + hi - b * B] = _nearest(new[:, h] / unit, cache)
            at += n
        return torch.from_numpy(codes) if cache == "e4m3" else None, torch.from_numpy(scale)

    k, k_scale = stored(rotated(st["k"]), st["k_cache"], st["k_scale"])
    v, v_scale = stored(st["v"].double().cpu().numpy(), st["v_cache"], st["v_scale"])
    return {"q": torch.from_numpy(rotated(st["q"])), "k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale}


def _exact_attend(case, st):
    rows, keys = _lengths(case)
    masks = _tree_bits(case, rows)
    H, KVH, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    g, at = H // KVH, 0
    out = torch.zeros(sum(rows), H, dim, dtype=torch.float64, device=DEV)
    for s, (n, K) in enumerate(zip(rows, keys)):
        base, slot = K - n, torch.arange(K, device=DEV)
        cells = st["table"][s].long()[slot // page], slice(None), slot % page
        units = cells[0], slice(None), slot % page // case["block"]
        k, v = (st[c].view(torch.uint8)[cells].view(st[c].dtype).float().double() * st[u][units].double()[..., None] for c, u in (("k_cache", "k_scale"), ("v_cache", "v_scale")))
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


def _exact_sample(case, st):
    logits = st["logits"].double().cpu().numpy()
    params = {name: None if st[name] is None else st[name].tolist() for name in ("uniform", "temperature", "top_k", "top_p", "min_p")}
    tokens, logprobs = [], []
    for r, x in enumerate(logits):
        T = params["temperature"][r]
        order = np.argsort(-x, kind="stable")
        if T <= 0:
            tokens.append(int(order[0]))
            logprobs.append(0.0)
            continue
        n = len(order)
        if params["top_k"] and params["top_k"][r] > 0:
            n = min(n, params["top_k"][r])
        w = np.exp((x[order[:n]] - x[order[0]]) / T)
        running = np.concatenate([[0.0], np.cumsum(w)])
        if params["top_p"] and params["top_p"][r] < 1:
            n = max(1, int(np.searchsorted(running, params["top_p"][r] * running[-1], side="left")))
        if params["min_p"] and params["min_p"][r] > 0:
            n = max(1, min(n, int((w >= params["min_p"][r]).sum())))
        n = min(n, len(w))
        i = min(n - 1, int(np.searchsorted(running[1:n + 1], params["uniform"][r] * running[n], side="right")))
        tokens.append(int(order[i]))
        logprobs.append(math.log(w[i] / running[n]) if w[i] > 0 else -math.inf)
    return {"token": torch.tensor(tokens, dtype=torch.int32), "logprob": torch.tensor(logprobs, dtype=torch.float64)}
