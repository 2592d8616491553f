"""Rotary positions and the append to a paged cache against the oracle in 64 bits.

Tolerances.  u = 2^-24.  A cosine or sine is the polynomial of an angle that is exact but for one rounding (angle at most pi / 4: u), the polynomial's own roundings
(3 u) and the factor mscale (u): 5 u of 1.  An element is two products and a sum of them: 5 u + 2 u + u of m (|a| + |b|).  What is stored in bf16 rounds once more, by
2^-8 of the value at most.  The oracle's angle (position * frequency in float64, positions below 2^22) is off by 2^22 * 2^-52."""
import numpy as np
import pytest
import torch

from oracle import operators as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def pkg():
    import paper_2401_15077_amd
    return paper_2401_15077_amd


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def test_rows_beyond_the_bound_are_left():
    """As in the attention: max_rows bounds the rows of a sequence that are processed."""
    p = pkg()
    k = torch.randn(5, 1, 8, device=DEV)
    q, before = k.clone(), k.clone()
    cache = torch.zeros(1, 1, 8, 8, device=DEV)
    kv = p.PagedKV(cache, cache.clone(), i32([[0], [0]]))
    p.rope(p.rope_plan(8), q, k, chunk=p.Chunk(i32([0, 3, 5]), i32([3, 5]), 5, 2, 8), kv=kv)
    assert torch.equal(q[2], before[2]) and not torch.equal(q[1], before[1]) and not torch.equal(q[4], before[4])
    assert float(cache[0, 0, 2].abs().sum()) == 0.0 and all(float(cache[0, 0, t].abs().sum()) > 0 for t in (0, 1, 3, 4))


def near(got, want, size, dtype, mscale=1.0):
    got = got.double().cpu().numpy()
    tol = 8 * U * size + (2.0 ** -8 * np.abs(want) * 1.001 if dtype == torch.bfloat16 else 0.0)
    worst = np.abs(got - want) / np.maximum(tol, 1e-30)
    assert worst.max() <= 1.0, worst.max()


def table_of(keys, page, spare=2, seed=0):
    need = [max(1, -(-k // page)) for k in keys]
    order = np.random.default_rng(seed).permutation(sum(need) + spare).tolist()
    t = np.full((len(keys), max(need) + 1), -1, np.int32)
    for s, n in enumerate(need):
        t[s, :n] = [order.pop() for _ in range(n)]
    return t, sum(need) + spare


CASES = [
    # rows, keys of each sequence, heads, kv heads, dim, rot, interleaved, scaling, page
    ([1], [1], 4, 4, 128, 128, False, "none", 64),
    ([1], [701], 32, 32, 128, 128, False, "none", 64),
    ([3, 1, 7], [3, 40, 130], 8, 2, 64, 64, True, "linear", 32),
    ([5, 2], [9, 65], 6, 3, 80, 40, False, "base", 16),
    ([4], [12], 5, 1, 80, 80, True, "ramp", 16),
    ([70, 33], [99, 33], 8, 2, 128, 64, True, "bands", 64),
    ([1100], [1300], 4, 2, 32, 32, False, "ramp", 128),
    ([2, 0, 3], [20, 5, 3], 3, 1, 20, 12, False, "none", 1),     # sizes that no 16-byte run divides
    ([6], [6], 2, 1, 6, 2, True, "none", 4),
    ([2], [7], 2, 2, 256, 256, False, "bands", 8),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
@pytest.mark.parametrize("types", ["fp32/fp32", "fp32/bf16", "bf16/bf16", "bf16/fp32"])
def test_rotation_and_append(case, types):
    rows, keys, H, KVH, D, rot, inter, scaling, page = case
    dtype, cdtype = (TYPES[t] for t in types.split("/"))
    p = pkg()
    gen = torch.Generator(device=DEV).manual_seed(7)
    R = sum(rows)
    q = torch.randn(R, H, D, device=DEV, generator=gen).to(dtype)
    k, v = (torch.randn(R, KVH, D, device=DEV, generator=gen).to(dtype) for _ in range(2))
    table, n_pages = table_of(keys, page)
    kc, vc = (torch.randn(n_pages, KVH, page, D, device=DEV, generator=gen).to(cdtype) for _ in range(2))
    kc0, vc0 = kc.clone(), vc.clone()
    start = np.cumsum([0] + rows)
    chunk = p.Chunk(i32(start.tolist()), i32(keys), R, max(rows), max(keys))
    kv = p.PagedKV(kc, vc, i32(table.tolist()))
    kw = dict(factor=1.0 if scaling == "none" else 8.0, low=1.0, high=32.0 if scaling == "ramp" else 4.0, trained_len=512)
    plan = p.rope_plan(D, theta=10000.0, rot_dim=rot, interleaved=inter, scaling=scaling, mscale=1.25, **kw)
    q_out = torch.full_like(q, 7.0)
    p.rope(plan, q, k, v, chunk=chunk, kv=kv, q_out=q_out)
    torch.cuda.synchronize()
    facts = ref.chunk_rows(start, keys)
    pos = [f[3] for f in facts]
    f = ref.frequencies(rot, scaling=scaling, **kw)
    want, size = ref.rotate(q.double().cpu().numpy(), pos, f, rot, inter, 1.25)
    near(q_out, want, size, dtype)
    want_k, size_k = ref.rotate(k.double().cpu().numpy(), pos, f, rot, inter, 1.25)
    touched = torch.zeros(n_pages, page, dtype=torch.bool, device=DEV)
    for r, s, t, _, _ in facts:
        pg, sl = table[s, t // page], t % page
        near(kc[pg, :, sl], want_k[r], size_k[r], cdtype)
        assert torch.equal(vc[pg, :, sl], v[r].to(cdtype))
        touched[pg, sl] = True
    # nothing else of the cache moved
    left = ~touched[:, None, :, None].expand_as(kc)
    assert torch.equal(kc[left], kc0[left]) and torch.equal(vc[left], vc0[left])
    # in place, without a cache: the same numbers
    q2, k2 = q.clone(), k.clone()
    p.rope(plan, q2, k2, chunk=chunk)
    assert torch.equal(q2, q_out)
    near(k2, want_k, size_k, dtype)
    # and with the positions given
    q3 = torch.empty_like(q)
    p.rope(plan, q, None, positions=i32(pos), q_out=q3)
    assert torch.equal(q3, q_out)


def test_tree_positions_and_places():
    p = pkg()
    masks = [0b1, 0b11, 0b101, 0b1011, 0b10101]
    base, page, H, KVH, D = [30, 4], 32, 4, 2, 64
    rows = [[0, 1, 3], [1, 2, 4]]                                 # rows of some of the nodes only, as in a pass over a tree level
    mask = torch.tensor([masks[u] for s in rows for u in s], dtype=torch.int64, device=DEV)
    table, n_pages = table_of([40, 40], page)
    kc = torch.zeros(n_pages, KVH, page, D, device=DEV)
    vc = torch.zeros_like(kc)
    chunk = p.Chunk(i32([0, 3, 6]), i32([35, 9]), 6, 3, 40, tree_base=i32(base), tree_mask=mask)
    k, v, q = torch.randn(6, KVH, D, device=DEV), torch.randn(6, KVH, D, device=DEV), torch.randn(6, H, D, device=DEV)
    q_out = torch.empty_like(q)
    p.rope(p.rope_plan(D), q, k, v, chunk=chunk, kv=p.PagedKV(kc, vc, i32(table.tolist())), q_out=q_out)
    f = ref.frequencies(D)
    r = 0
    for s in range(2):
        for u in rows[s]:
            pos, token = base[s] + bin(masks[u]).count("1") - 1, base[s] + u
            want, size = ref.rotate(k[r:r + 1].double().cpu().numpy(), [pos], f, D, False)
            near(kc[table[s, token // page], :, token % page][None], want, size, torch.float32)
            assert torch.equal(vc[table[s, token // page], :, token % page], v[r])
            want, size = ref.rotate(q[r:r + 1].double().cpu().numpy(), [pos], f, D, False)
            near(q_out[r:r + 1], want, size, torch.float32)
            r += 1
    assert int((vc != 0).any(-1).any(1).sum()) == 6


@pytest.mark.parametrize("position", [0, 1, 4095, 2 ** 20 + 7, 2 ** 30 + 12345, 2 ** 31 - 1, -5])
def test_far_positions_lose_nothing(position):
    """Angles modulo a turn from exact rational arithmetic: position * (frequency / 2 pi) with 60 digits."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
    p = pkg()
    D = 64
    x = torch.randn(1, 1, D, device=DEV)
    out = torch.empty_like(x)
    p.rope(p.rope_plan(D, theta=500000.0), x, None, positions=i32([position]), q_out=out)
    a = x.double().cpu().numpy()[0, 0]
    got = out.double().cpu().numpy()[0, 0]
    for i in range(D // 2):
        f = (Decimal(500000).ln() * (Decimal(-2 * i) / D)).exp()
        turns = f * position / (2 * pi)
        ang = float((turns - turns.to_integral_value()) * 2 * pi)
        c, s = np.cos(ang), np.sin(ang)
        # the frequency is held to 2^-65 turn: at 2^31 positions 2^-34 turn, 2^-31.3 rad
        tol = (8 * U + 2.0 ** -31) * (abs(a[i]) + abs(a[i + D // 2]))
        assert abs(got[i] - (a[i] * c - a[i + D // 2] * s)) <= tol
        assert abs(got[i + D // 2] - (a[i + D // 2] * c + a[i] * s)) <= tol


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_transposed_map_is_the_gradient(inter, dtype):
    """y = rope(x): the gradient of <w, y> is the transposed map of w, as the formula has it and by differences in 64 bits."""
    p = pkg()
    D, rot, R = 32, 24, 9
    plan = p.rope_plan(D, rot_dim=rot, interleaved=inter, scaling="linear", factor=3.0, mscale=0.7)
    w = torch.randn(R, 3, D, device=DEV).to(TYPES[dtype])
    pos = list(range(100, 100 + R))
    g = torch.empty_like(w)
    p.rope(plan, w, None, positions=i32(pos), q_out=g, inverse=True)
    f = ref.frequencies(rot, scaling="linear", factor=3.0)
    wn = w.double().cpu().numpy()
    want, size = ref.rotate(wn, pos, f, rot, inter, 0.7, inverse=True)
    near(g, want, size, w.dtype)
    x = np.random.default_rng(0).standard_normal(wn.shape)
    for r, h, e in ((0, 0, 0), (3, 1, 5), (8, 2, rot - 1), (4, 0, D - 1)):
        d = np.zeros_like(x)
        d[r, h, e] = 1e-3
        diff = ((ref.rotate(x + d, pos, f, rot, inter, 0.7)[0] - ref.rotate(x - d, pos, f, rot, inter, 0.7)[0]) * wn).sum() / 2e-3
        assert abs(diff - want[r, h, e]) < 1e-9


def test_strided_and_unaligned_tensors():
    """q, k, v as views of one fused projection; rows that begin off 16-byte pieces; caches with another order of heads and tokens."""
    p = pkg()
    H, KVH, D, R, page = 4, 2, 64, 5, 16
    plan = p.rope_plan(D)
    pos = i32(list(range(11, 11 + R)))
    base = torch.randn(R, (H + 2 * KVH) * D, device=DEV)
    want = torch.empty(R, H, D, device=DEV)
    p.rope(plan, base[:, :H * D].reshape(R, H, D).contiguous(), None, positions=pos, q_out=want)
    fused = base.clone()
    p.rope(plan, fused[:, :H * D].view(R, H, D), None, positions=pos)
    assert torch.equal(fused[:, :H * D].view(R, H, D), want) and torch.equal(fused[:, H * D:], base[:, H * D:])
    odd = torch.zeros(R * (H * D + 3) + 1, device=DEV)
    view = odd[1:].view(R, H * D + 3)[:, :H * D].unflatten(1, (H, D))
    view.copy_(base[:, :H * D].view(R, H, D))
    p.rope(plan, view, None, positions=pos)
    assert torch.equal(view, want)
    # a cache laid out [page][token][head][dim]
    store = torch.zeros(3, page, KVH, D, device=DEV), torch.zeros(3, page, KVH, D, device=DEV)
    kv = p.PagedKV(store[0].transpose(1, 2), store[1].transpose(1, 2), i32([[2, 0]]))
    chunk = p.Chunk(i32([0, R]), i32([18]), R, R, 32)
    k, v = base[:, H * D:(H + KVH) * D].view(R, KVH, D), base[:, (H + KVH) * D:].view(R, KVH, D)
    p.rope(plan, None, k, v, chunk=chunk, kv=kv)
    kk = torch.empty(R, KVH, D, device=DEV)
    p.rope(plan, None, k.contiguous(), positions=i32(list(range(13, 18))), k_out=kk)
    got = torch.stack([store[0][2 if t < page else 0, t % page] for t in range(13, 18)])
    assert torch.equal(got, kk)
    assert torch.equal(torch.stack([store[1][2 if t < page else 0, t % page] for t in range(13, 18)]), v)


def test_rows_of_no_sequence_and_pages_that_are_not_there():
    p = pkg()
    H, KVH, D, page = 2, 1, 32, 8
    q, k, v = torch.randn(6, H, D, device=DEV), torch.randn(6, KVH, D, device=DEV), torch.randn(6, KVH, D, device=DEV)
    kc, vc = torch.full((2, KVH, page, D), 3.0, device=DEV), torch.full((2, KVH, page, D), 3.0, device=DEV)
    q_out = torch.full_like(q, 9.0)
    # rows 0 and 5 belong to nobody; sequence 0's token 8 would be on page -1, sequence 1's tokens at or behind max_keys
    chunk = p.Chunk(i32([1, 3, 5]), i32([9, 20]), 6, 4, 16)
    p.rope(p.rope_plan(D), q, k, v, chunk=chunk, kv=p.PagedKV(kc, vc, i32([[0, -1, 1], [1, 7, 1]])), q_out=q_out)
    assert torch.all(q_out[0] == 9.0) and torch.all(q_out[5] == 9.0)
    want, size = ref.rotate(q[1:5].double().cpu().numpy(), [7, 8, 18, 19], ref.frequencies(D), D, False)
    near(q_out[1:5], want, size, torch.float32)
    assert torch.equal(vc[0, :, 7], v[1])
    vc[0, :, 7] = 3.0
    kc[0, :, 7] = 3.0
    assert torch.all(vc == 3.0) and torch.all(kc == 3.0)
    p.rope(p.rope_plan(D), q[:0], k[:0], v[:0], chunk=p.Chunk(i32([0, 0, 0]), i32([0, 0]), 0, 1, 1), kv=p.PagedKV(kc, vc, i32([[0], [1]])))
