"""Outputs that lie on part of what a call reads are refused before anything is launched (addresses are never followed); outputs that are the input, or lie beside it in one buffer, are not."""
import itertools

import numpy as np
import pytest
import torch

import paper_2401_15077_amd as pkg
from paper_2401_15077_amd import operators as ops

A, EINVAL = 1 << 20, -1


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2401_15077_amd import build
        build.build()
    return pkg.load_library()


def chunk(n):
    return ops.EagleChunk(n_seqs=1, n_rows=n, max_rows=n, max_keys=100, row_start=A, key_len=A)


def paged(heads, dim):
    return ops.EaglePagedKV(k=A << 20, v=A << 21, dtype=1, n_kv_heads=heads, head_dim=dim, page_tokens=32, n_pages=9, pages_per_seq=4, page_stride=heads * 32 * dim, head_stride=32 * dim,
                            token_stride=dim, table_stride=4, page_table=A)


def cells(at, rows, row, heads, head, dim):
    return {at + r * row + h * head + i for r, h, i in itertools.product(range(rows), range(heads), range(dim))}


def accepted(lib, out, q, rows, heads, dim, strides, out_strides=None):
    """Whether the attention takes these (element) offsets; its workspace call makes the same checks and launches nothing."""
    so = out_strides or strides
    a = ops.EagleAttentionArgs(n_heads=heads, dtype=1, q=A + 2 * q, out=A + 2 * out, q_row=strides[0], q_head=strides[1], out_row=so[0], out_head=so[1], scale=0.1)
    return lib.eagle_chunk_attention_workspace(a, chunk(rows), paged(heads, dim)) > 0


@pytest.mark.parametrize("rows,heads,dim,strides", [(3, 2, 8, (16, 8)), (3, 2, 8, (48, 8)), (3, 2, 8, (8, 24)), (1, 4, 8, (8, 16)), (4, 1, 16, (32, 8)), (5, 3, 8, (40, 16)), (2, 2, 16, (16, 32)),
                                                   (1, 1, 24, (8, 8)), (6, 2, 8, (8, 56))])
def test_equal_strides_are_judged_exactly(lib, rows, heads, dim, strides):
    span = rows * abs(strides[0]) + heads * abs(strides[1]) + dim
    for apart in range(-span - 16, span + 17, 8):
        common = cells(0, rows, strides[0], heads, strides[1], dim) & cells(apart, rows, strides[0], heads, strides[1], dim)
        assert accepted(lib, 4096 + apart, 4096, rows, heads, dim, strides) == (apart == 0 or not common), apart


def test_strides_of_a_single_row_or_head_do_not_count(lib):
    assert accepted(lib, 0, 0, 1, 4, 8, (32, 8), (640, 8))        # one row: the same place whatever the row stride
    assert accepted(lib, 0, 0, 4, 1, 8, (32, 8), (32, 80))
    assert not accepted(lib, 8, 0, 1, 4, 8, (32, 8), (640, 8))
    assert not accepted(lib, 32, 0, 4, 1, 8, (32, 8), (32, 80))


def test_rope(lib):
    good = dict(n_rows=4, n_heads=4, n_kv_heads=2, dtype=0, q=A, k=A + (1 << 16), q_out=A + (2 << 16), k_out=A + (3 << 16), q_row=256, q_head=64, k_row=128, k_head=64, q_out_row=256,
                q_out_head=64, k_out_row=128, k_out_head=64, positions=A)
    bad = [dict(q_out=A + 4), dict(q_out=A + 256), dict(k_out=A + (1 << 16) + 512), dict(q_out=A + (1 << 16), q_out_row=128), dict(k_out=A, k_out_row=256, k_row=256),
           dict(k_out=A + (2 << 16), k_out_row=256), dict(k=A, k_row=256, q_out=A)]
    for kw in bad:
        a = ops.EagleRopeArgs(**{**good, **kw})
        assert lib.eagle_rope(pkg.rope_plan(64), a, None, None, None) == EINVAL, kw
        assert b"lies on" in lib.eagle_last_error(), kw


def test_logit_rules(lib):
    good = dict(n_rows=4, vocab=100, dtype=0, in_=A, out=A, in_stride=128, out_stride=128)
    for kw in (dict(out=A + 4), dict(out=A + 399), dict(out=A + 512), dict(out=A - 3 * 512), dict(out=A + 512 + 112 + 4)):
        assert lib.eagle_apply_logit_rules(ops.EagleLogits(**{**good, **kw}), ops.EagleLogitRules(n_seqs=4), None) == EINVAL, kw
        assert b"out lies on part of in" in lib.eagle_last_error(), kw


# ----------------------------------------------------------------------------- and what stays allowed
DEV = "cuda:0"


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


@pytest.mark.gpu
def test_tensors_side_by_side_in_one_buffer():
    gen = torch.Generator(device=DEV).manual_seed(3)
    R, H, KVH, D, V = 7, 4, 2, 64, 130
    packed = torch.randn(R, H + 2 * KVH + H + KVH, D, device=DEV, generator=gen)
    q, k, v, q2, k2 = packed[:, :H], packed[:, H:H + KVH], packed[:, H + KVH:H + 2 * KVH], packed[:, H + 2 * KVH:2 * H + 2 * KVH], packed[:, 2 * H + 2 * KVH:]
    plan, at = pkg.rope_plan(D), i32(range(R))
    want_q, want_k = torch.empty(R, H, D, device=DEV), torch.empty(R, KVH, D, device=DEV)
    pkg.rope(plan, q.clone(), k.clone(), positions=at, q_out=want_q, k_out=want_k)
    pkg.rope(plan, q, k, positions=at, q_out=q2, k_out=k2)
    assert torch.equal(q2, want_q) and torch.equal(k2, want_k)
    c = pkg.Chunk(i32([0, R]), i32([40]), R, R, 40)
    kc, vc = (torch.randn(2, KVH, 32, D, device=DEV, generator=gen) for _ in range(2))
    kv = pkg.PagedKV(kc, vc, i32([[0, 1]]))
    want = pkg.chunk_attention(q.clone(), kv, c)
    assert torch.equal(pkg.chunk_attention(q, kv, c, out=q2), want)
    one = packed[:1, :H]                                          # a single row: its row stride differs from the output's and does not matter
    c1 = pkg.Chunk(i32([0, 1]), i32([40]), 1, 1, 40)
    want = pkg.chunk_attention(one.clone(), kv, c1)
    assert torch.equal(pkg.chunk_attention(one, kv, c1, out=packed[:1, H + 2 * KVH:2 * H + 2 * KVH]), want)
    pkg.rope(plan, q, k, v, chunk=c, kv=kv, positions=at)         # in place, q, k and v in one buffer
    assert torch.equal(q, want_q)
    x = torch.randn(R, 2 * V, device=DEV, generator=gen)
    r = pkg.LogitRules(n_seqs=R, bias=(i32(range(R + 1)), i32([5] * R), torch.ones(R, device=DEV)))
    want = pkg.apply_logit_rules(x[:, :V].clone(), r)
    assert torch.equal(pkg.apply_logit_rules(x[:, :V], r, out=x[:, V:]), want)
    assert torch.equal(pkg.apply_logit_rules(x[:, :V], r), want)
