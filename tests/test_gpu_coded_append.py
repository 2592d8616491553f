"""Rotation with the append to a paged cache of 8-bit codes against the oracle in 64 bits.

Codes and scales are worked out in 64 bits and rounded once, so they have to be the oracle's, but where the oracle's own number lies within 2^-40 of a border between two codes (positions below
2^22, an angle's error 2^22 * 2^-52, times elements of a few units): there a neighbour is right too, and no more than one element in 10^5 may lie so.  Queries: as in test_gpu_rope.py."""
import numpy as np
import pytest
import torch

from oracle import operators as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def pkg():
    import paper_2401_15077_amd
    return paper_2401_15077_amd


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def numbers(codes):
    return ref.code_value(codes.view(torch.uint8).cpu().numpy(), codes.dtype == torch.float8_e4m3fn)


def random_cache(gen, n_pages, KVH, page, D, cache, block, pad=0):
    """Codes of all kinds but NaN, scales that are no powers of two."""
    c = torch.randint(0, 256, (n_pages, KVH, page, D + pad), device=DEV, generator=gen, dtype=torch.int32)
    if cache == "e4m3":
        c = torch.where(c & 127 == 127, c - 1, c)
    else:
        c = torch.where(c == 128, 127, c)
    c = c.to(torch.uint8).view(CODES[cache])[..., :D]
    return c, torch.rand(n_pages, KVH, page // block, device=DEV, generator=gen) * 0.02 + 0.0005


def compare(got, got_scale, want, want_scale, exact, e4m3):
    np.testing.assert_array_equal(got_scale.double().cpu().numpy(), want_scale)
    got = numbers(got)
    off = ~((got == want) | (np.isnan(got) & np.isnan(want)))
    if off.any():
        x = exact[off]
        assert (np.abs(ref.nearest_code(x * (1 + 2.0 ** -40), e4m3) - ref.nearest_code(x * (1 - 2.0 ** -40), e4m3)) > 0).all(), (got[off][:5], want[off][:5], x[:5])
        assert off.sum() <= 1e-5 * off.size, off.sum()


def run(rows, keys, H, KVH, D, dtype, cache, page, block, *, rot=None, inter=False, masks=None, base=None, positions=None, v=True, max_rows=None, max_keys=None, gap=(), pad=0, change=None, mscale=1.0,
        seed=0, scales=None, spread=False):
    p = pkg()
    rot = rot or D
    gen = torch.Generator(device=DEV).manual_seed(seed + 11)
    R, S = sum(rows), len(rows)
    need = [max(1, -(-k // page)) for k in keys]
    n_pages = sum(need) + 2
    order = np.random.default_rng(seed).permutation(n_pages).tolist()
    table = np.full((S, max(need) + 1), -3, np.int32)
    for s, n in enumerate(need):
        table[s, :n] = [order.pop() for _ in range(n)]
    for s, g in gap:
        table[s, g] = n_pages + 1 if g % 2 else -1
    kc, ks = random_cache(gen, n_pages, KVH, page, D, cache, block, pad)
    vc, vs = random_cache(gen, n_pages, KVH, page, D, cache, block, pad)
    if scales is not None:
        ks.copy_(scales(ks)), vs.copy_(scales(vs))
    q = torch.randn(R, H, D, device=DEV, generator=gen).to(TYPES[dtype])
    k, val = ((torch.randn(R, KVH, D, device=DEV, generator=gen) * torch.exp(torch.randn(R, KVH, 1, device=DEV, generator=gen))).to(TYPES[dtype]) for _ in range(2))
    if change is not None:
        change(k), change(val)
    if spread:                                                    # rows and heads of wider tensors
        q, k, val = (torch.cat([t, t], 2).transpose(0, 1).contiguous().transpose(0, 1)[:, :, :D] for t in (q, k, val))
    start = np.cumsum([0] + list(rows))
    tm = None if masks is None else torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device=DEV)
    mr, mk = max_rows or max(max(rows), 1), max_keys or max(keys) + 3
    chunk = p.Chunk(i32(start), i32(keys), R, mr, mk, tree_base=None if base is None else i32(base), tree_mask=tm)
    kv = p.PagedKV8(kc, vc, i32(table), ks, vs)
    plan = p.rope_plan(D, rot_dim=rot, interleaved=inter, mscale=mscale)
    before = [(numbers(c), s.double().cpu().numpy()) for c, s in ((kc, ks), (vc, vs))]
    bytes_before = [c.contiguous().view(torch.uint8).clone() for c in (kc, vc)]
    q_out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    p.rope(plan, q, k, val if v else None, chunk=chunk, kv=kv, positions=None if positions is None else i32(positions), q_out=q_out)
    torch.cuda.synchronize()
    facts = ref.chunk_rows(start, keys, base, masks)
    pos = [f[3] for f in facts] if positions is None else positions
    freqs = ref.frequencies(rot)
    turned, _ = ref.rotate(k.double().cpu().numpy(), pos, freqs, rot, inter, float(np.float32(mscale)))
    kw = dict(page=page, block=block, e4m3=cache == "e4m3", max_rows=mr, max_keys=mk, row_start=start)
    for i, (x, c, s) in enumerate(((turned, kc, ks), (val.double().cpu().numpy(), vc, vs))):
        if i and not v:
            assert torch.equal(c.contiguous().view(torch.uint8), bytes_before[1])
            np.testing.assert_array_equal(s.double().cpu().numpy(), before[1][1])
            continue
        want = ref.append_codes(x, *before[i], facts, table, keys, **kw)
        compare(c, s, *want, cache == "e4m3")
    wq, size = ref.rotate(q.double().cpu().numpy(), pos, freqs, rot, inter, float(np.float32(mscale)))
    skipped = np.array([r - start[s] >= mr for r, s, *_ in facts], dtype=bool)
    tol = 8 * U * size + (2.0 ** -8 * np.abs(wq) * 1.001 if dtype == "bf16" else 0.0) + 1e-30
    got = q_out.double().cpu().numpy()
    assert (np.abs(got - wq) <= tol)[~skipped].all()
    assert (got[skipped] == 7.0).all()
    return kv


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,keys,H,KVH,D,rot,inter,page,block", [
    ([1], [1], 4, 4, 128, 128, False, 64, 16), ([1], [701], 8, 8, 128, 128, False, 64, 16), ([1], [16], 2, 1, 64, 64, True, 16, 16), ([1], [17], 2, 1, 64, 32, True, 16, 16),
    ([3, 1, 0, 7], [3, 40, 9, 130], 8, 2, 64, 64, True, 32, 32), ([5, 2], [9, 65], 6, 3, 80, 40, False, 128, 64), ([70, 33], [99, 33], 8, 2, 128, 64, True, 128, 128),
    ([300], [523], 4, 2, 32, 32, False, 64, 64), ([130, 64], [130, 1000], 3, 1, 256, 256, False, 256, 128), ([2, 0, 3], [20, 5, 3], 3, 1, 20, 12, False, 16, 16),
    ([40], [60], 2, 1, 6, 2, True, 32, 16), ([1] * 70, list(range(1, 71)), 4, 2, 64, 64, False, 32, 16),
])
def test_rotation_and_append(rows, keys, H, KVH, D, rot, inter, page, block, dtype, cache):
    run(rows, keys, H, KVH, D, dtype, cache, page, block, rot=rot, inter=inter, mscale=1.25)


def tree(n, rng):
    masks, depth = [1], [0]
    for v in range(1, n):
        p = int(rng.choice([u for u in range(v) if depth[u] < 15]))
        masks.append(masks[p] | 1 << v)
        depth.append(depth[p] + 1)
    return masks


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("nodes,base", [([26], [674]), ([26, 8, 1], [100, 0, 63]), ([64], [15]), ([64, 64], [31, 17])])
def test_trees(nodes, base, cache):
    rng = np.random.default_rng(sum(nodes))
    masks = [m for n in nodes for m in tree(n, rng)]
    for block in (16, 64):
        run(nodes, [b + n for b, n in zip(base, nodes)], 4, 2, 64, "fp32", cache, 64, block, masks=masks, base=base)


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
def test_some_nodes_of_a_tree(cache):
    """A level of two trees: nodes without a row here are other tokens of their blocks."""
    rng = np.random.default_rng(5)
    t = [tree(26, rng), tree(15, rng)]
    masks = [t[0][u] for u in (1, 2, 5, 9)] + [t[1][u] for u in (3, 4)]
    run([4, 2], [126, 45], 8, 2, 64, "bf16", cache, 32, 16, masks=masks, base=[100, 30])
    # and a row that is no node
    run([4, 2], [126, 45], 8, 2, 64, "bf16", cache, 32, 32, masks=masks[:3] + [t[0][9]] + masks[4:], base=[100, 30], positions=[5, 6, 7, 70000, 1, 0])


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("kw", [dict(max_rows=3), dict(max_keys=50), dict(v=False), dict(gap=[(0, 1), (1, 0)]), dict(positions=list(range(90000, 90029))), dict(pad=16), dict(pad=3),
                                dict(spread=True)], ids=str)
def test_bounds_gaps_positions_and_strides(kw, cache):
    run([20, 9], [70, 40], 4, 2, 64, "fp32", cache, 32, 16, **kw)
    run([20, 9], [70, 40], 4, 2, 64, "bf16", cache, 64, 32, **kw)


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("v", [False, True])
def test_more_than_4096_work_groups(v, inter, dtype, cache):
    """Those that append are spread among those that rotate queries."""
    run([1300, 1, 900], [1310, 77, 900], 2, 16 if v else 32, 16, dtype, cache, 64, 16, inter=inter, v=v)


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("scale", [0.0, -0.01, float("inf"), float("nan"), 2.0 ** -140, 3e38, 2.0 ** 100, 1.5 * 2.0 ** 99])
def test_scales_of_all_kinds(scale, cache):
    run([1, 40], [40, 70], 2, 2, 64, "fp32", cache, 64, 32, scales=lambda s: torch.full_like(s, scale))


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("size", [0.0, 1e-44, 1e-38, 1e30, 3e38])
def test_sizes_of_all_kinds(size, cache):
    run([3, 40], [40, 70], 2, 2, 64, "fp32", cache, 64, 32, change=lambda x: x.clamp_(-1.0, 1.0).mul_(size))


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_what_is_not_finite(dtype, cache):
    """Of a value; a key's rotation would spread it over the pair as the definition says."""
    def spoil(x):
        x[0, 0, 3], x[1, 1, 5], x[2, 0, 7], x[30, 0] = float("nan"), float("inf"), float("-inf"), float("nan")
    p = pkg()
    gen = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn(43, 2, 64, device=DEV, generator=gen).to(TYPES[dtype]) for _ in range(2))
    spoil(v)
    kc, ks = random_cache(gen, 4, 2, 64, 64, cache, 32)
    vc, vs = random_cache(gen, 4, 2, 64, 64, cache, 32)
    before = numbers(vc), vs.double().cpu().numpy()
    table = np.array([[1, 2], [0, 3]])
    p.rope(p.rope_plan(64), None, k, v, chunk=p.Chunk(i32([0, 3, 43]), i32([40, 70]), 43, 40, 70), kv=p.PagedKV8(kc, vc, i32(table), ks, vs))
    facts = ref.chunk_rows([0, 3, 43], [40, 70])
    want = ref.append_codes(v.double().cpu().numpy(), *before, facts, table, [40, 70], page=64, block=32, e4m3=cache == "e4m3", max_rows=40, max_keys=70, row_start=[0, 3, 43])
    compare(vc, vs, *want, cache == "e4m3")


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
def test_ties(cache):
    """Values half-way between two codes, under a scale that is no power of two and one that is, and codes that are halved to half-way."""
    p = pkg()
    M = 448.0 if cache == "e4m3" else 127.0
    codes = torch.arange(0, 256, dtype=torch.int32).to(torch.uint8)
    n = np.unique(ref.code_value(codes.numpy(), cache == "e4m3"))
    n = n[np.isfinite(n) & (np.abs(n) <= M)]
    half = (n[1:] + n[:-1]) / 2
    half = half[np.abs(half) < M]
    D = 256
    for s in (3 * 2.0 ** -5, 2.0 ** -3):
        row = np.zeros(D)
        row[:len(half)] = half * s
        v = torch.tensor(row, dtype=torch.float32, device=DEV).view(1, 1, D)
        assert (v.double().cpu().numpy().ravel() == row).all()
        kc, vc = (torch.zeros(1, 1, 16, D, device=DEV, dtype=torch.uint8) for _ in range(2))
        vc[0, 0, 0] = torch.where(codes & 127 == 127 if cache == "e4m3" else codes == 128, torch.zeros_like(codes), codes).to(DEV)
        kc, vc = kc.view(CODES[cache]), vc.view(CODES[cache])
        ks, vs = (torch.full((1, 1, 1), s, device=DEV) for _ in range(2))
        for double in (1.0, 2.0):                                 # the second time the scale doubles, and the codes in the cache are halved
            if double > 1:
                v = v.clone()
                v[0, 0, -1] = 1.9 * M * s
            before = numbers(vc), vs.double().cpu().numpy()
            at = 1 if double == 1 else 2
            p.rope(p.rope_plan(D), None, torch.zeros_like(v), v, chunk=p.Chunk(i32([0, 1]), i32([at + 1]), 1, 1, 16), kv=p.PagedKV8(kc, vc, i32([[0]]), ks, vs))
            want = ref.append_codes(v.double().cpu().numpy(), *before, ref.chunk_rows([0, 1], [at + 1]), [[0]], [at + 1], page=16, block=16, e4m3=cache == "e4m3", max_rows=1, max_keys=16, row_start=[0, 1])
            np.testing.assert_array_equal(numbers(vc), want[0])
            np.testing.assert_array_equal(vs.double().cpu().numpy(), want[1])


def test_the_same_bits_every_time():
    a, b = (run([26, 300], [200, 400], 8, 2, 128, "bf16", "e4m3", 64, 32) for _ in range(2))
    for x, y in zip(a.both, b.both):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
