"""What the operators on the caller's own tensors refuse, before anything is launched: at the C entry (no GPU needed: the addresses are never followed) and in
the binding."""
import ctypes

import pytest
import torch

import paper_2401_15077_amd as pkg
from paper_2401_15077_amd import operators as ops

A = 1 << 20                                                       # an address, never followed
EINVAL, ENOMEM = -1, -2


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2401_15077_amd import build
        build.build()
    return pkg.load_library()


def chunk(**kw):
    return ops.EagleChunk(**{**dict(n_seqs=2, n_rows=4, max_rows=3, max_keys=100, row_start=A, key_len=A), **kw})


def paged(**kw):
    return ops.EaglePagedKV(**{**dict(k=A, v=A, dtype=1, n_kv_heads=2, head_dim=64, page_tokens=32, n_pages=9, pages_per_seq=4, page_stride=2 * 32 * 64, head_stride=32 * 64, token_stride=64,
                                      table_stride=4, page_table=A), **kw})


def plan():
    return pkg.rope_plan(64)


BAD_CHUNKS = [dict(n_seqs=0), dict(n_rows=-1), dict(max_rows=0), dict(max_keys=0), dict(row_start=None), dict(key_len=None), dict(tree_base=A), dict(tree_mask=A)]
BAD_CACHES = [dict(k=None), dict(v=None), dict(page_table=None), dict(dtype=2), dict(n_kv_heads=0), dict(page_tokens=0), dict(page_tokens=24), dict(n_pages=0), dict(pages_per_seq=0),
              dict(page_stride=0), dict(head_stride=-64), dict(token_stride=0), dict(table_stride=3)]


@pytest.mark.parametrize("kw", [dict(head_dim=0), dict(head_dim=258), dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=66), dict(scaling=5), dict(scaling=-1), dict(theta=1.0),
                                dict(theta=float("nan")), dict(theta=float("inf")), dict(mscale=float("inf")), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")),
                                dict(scaling=2, factor=2.0, rot_dim=2), dict(scaling=3, factor=2.0, low=0.0), dict(scaling=3, factor=2.0, low=4.0, high=4.0),
                                dict(scaling=4, factor=2.0, trained_len=0), dict(scaling=4, factor=2.0, high=float("inf"))], ids=str)
def test_rope_plan(lib, kw):
    cfg = ops.EagleRopeConfig(**{**dict(head_dim=64, rot_dim=64, theta=1e4, factor=1.0, low=1.0, high=4.0, trained_len=4096, mscale=1.0), **kw})
    assert lib.eagle_rope_plan_init(ctypes.byref(cfg), ctypes.byref(ops.EagleRopePlan())) == EINVAL
    assert lib.eagle_last_error()


def test_rope(lib):
    good = dict(n_rows=4, n_heads=4, n_kv_heads=2, dtype=1, q=A, k=A, v=A, q_out=A, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, q_out_row=256, q_out_head=64)

    def call(p=None, c=None, kv=None, **kw):
        return lib.eagle_rope(plan() if p is None else p, ops.EagleRopeArgs(**{**good, **kw}), c, kv, None)

    assert call(c=chunk(), kv=paged(), dtype=2) == EINVAL
    assert call(c=chunk(), kv=paged(), n_rows=-1) == EINVAL
    assert call(c=chunk(), kv=paged(), n_rows=5) == EINVAL                     # the chunk has 4
    assert call(c=chunk(), kv=paged(), q=None, k=None) == EINVAL
    assert call(c=chunk(), kv=paged(), q_out=None) == EINVAL
    assert call(c=chunk(), kv=paged(), k=None) == EINVAL
    assert call(c=chunk(), kv=paged(), k_out=A) == EINVAL
    assert call(c=chunk(), kv=paged(), inverse=1) == EINVAL
    assert call(c=chunk(), kv=paged(), n_kv_heads=4) == EINVAL
    assert call(c=chunk(), kv=paged(head_dim=128)) == EINVAL
    assert call(kv=paged(), positions=A) == EINVAL                             # a cache needs a chunk
    assert call(v=None, k_out=A) == EINVAL                                     # no positions
    assert call(c=chunk(), k_out=A) == EINVAL                                  # v without a cache
    assert call(c=chunk(), v=None) == EINVAL                                   # k goes nowhere
    assert call(p=ops.EagleRopePlan(), c=chunk(), kv=paged()) == EINVAL
    assert lib.eagle_rope(None, None, None, None, None) == EINVAL
    for bad in BAD_CHUNKS:
        assert call(c=chunk(**bad), kv=paged()) == EINVAL, bad
    for bad in BAD_CACHES:
        assert call(c=chunk(), kv=paged(**bad)) == EINVAL, bad


def test_attention(lib):
    good = dict(n_heads=4, dtype=1, q=A, out=A, q_row=256, q_head=64, out_row=256, out_head=64, scale=0.1)

    def call(c=None, kv=None, ws=A, size=1 << 40, **kw):
        a, c, kv = ops.EagleAttentionArgs(**{**good, **kw}), c or chunk(), kv or paged()
        rc = lib.eagle_chunk_attention(a, c, kv, ws, size, None)
        if ws == A and size == 1 << 40:
            assert (lib.eagle_chunk_attention_workspace(a, c, kv) == 0) == (rc == EINVAL)
        return rc

    for kw in (dict(dtype=3), dict(n_heads=0), dict(n_heads=3), dict(q=None), dict(out=None), dict(scale=float("nan")), dict(softcap=-1.0), dict(softcap=float("inf")),
               dict(window=-1), dict(q=A + 8), dict(out=A + 8), dict(q_row=252), dict(q_head=60), dict(out_row=260), dict(out_head=68)):
        assert call(**kw) == EINVAL, kw
    for kv in (dict(head_dim=136), dict(head_dim=60), dict(dtype=0), dict(k=A + 4), dict(v=A + 4), dict(token_stride=68), dict(head_stride=2044), dict(page_stride=4100)):
        assert call(kv=paged(**kv)) == EINVAL, kv
    for bad in BAD_CHUNKS:
        assert call(c=chunk(**bad)) == EINVAL, bad
    for bad in BAD_CACHES:
        assert call(kv=paged(**bad)) == EINVAL, bad
    assert call(ws=None) == EINVAL and call(ws=A + 64) == EINVAL
    need = lib.eagle_chunk_attention_workspace(ops.EagleAttentionArgs(**good), chunk(), paged())
    assert need > 0 and call(size=need - 1) == ENOMEM
    assert lib.eagle_chunk_attention(None, None, None, None, 0, None) == EINVAL


def test_logit_rules(lib):
    good = dict(n_rows=4, vocab=100, dtype=0, in_=A, out=A, in_stride=100, out_stride=100, row_start=A)

    def call(rules=None, **kw):
        return lib.eagle_apply_logit_rules(ops.EagleLogits(**{**good, **kw}), ops.EagleLogitRules(**{**dict(n_seqs=2), **(rules or {})}), None)

    for kw in (dict(dtype=2), dict(n_rows=-1), dict(vocab=0), dict(in_=None), dict(out=None), dict(in_stride=99), dict(out_stride=99), dict(row_start=None), dict(path_token=A), dict(path_mask=A),
               dict(allowed=A), dict(allowed=A, n_masks=1, mask_stride=3)):
        assert call(**kw) == EINVAL, kw
    for r in (dict(n_seqs=0), dict(tokens=A), dict(tokens=A, n_tokens=A, token_stride=-1), dict(bias_token=A), dict(bias_token=A, bias_start=A), dict(bias_token=A, bias_start=A, bias_value=A, n_bias=-1)):
        assert call(r) == EINVAL, r
    assert lib.eagle_apply_logit_rules(None, None, None) == EINVAL


# ----------------------------------------------------------------------------- the binding
def i32(*a):
    return torch.tensor(a, dtype=torch.int32)


def test_binding_checks():
    R, S = 4, 2
    k = torch.zeros(9, 2, 32, 64)
    kv = pkg.PagedKV(k, k.clone(), torch.zeros(S, 4, dtype=torch.int32))
    c = pkg.Chunk(i32(0, 2, 4), i32(5, 6), R, 2, 10)
    q, kk = torch.zeros(R, 4, 64), torch.zeros(R, 2, 64)
    with pytest.raises(ValueError, match="scaling"):
        pkg.rope_plan(64, scaling="other")
    with pytest.raises(ValueError, match="row_start"):
        pkg.Chunk(i32(0, 2), i32(5, 6), R, 2, 10)
    with pytest.raises(ValueError, match="tree_mask"):
        pkg.Chunk(i32(0, 2, 4), i32(5, 6), R, 2, 10, tree_base=i32(0, 0), tree_mask=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="row_start"):
        pkg.Chunk(torch.zeros(3, dtype=torch.int64), i32(5, 6), R, 2, 10)
    for bad in ((k, k[:8]), (k, k.bfloat16()), (k.double(), k.double()), (k, k.transpose(1, 2).contiguous().transpose(1, 2)), (k[..., ::2], k[..., ::2])):
        with pytest.raises(ValueError, match="k and v|consecutive"):
            pkg.PagedKV(*bad, torch.zeros(S, 4, dtype=torch.int32))
    with pytest.raises(ValueError, match="page_table"):
        pkg.PagedKV(k, k, torch.zeros(S, 4, dtype=torch.int64))
    p = plan()
    for args, kw in (((q[..., :32], kk), {}), ((q, kk[:3]), {}), ((q, kk.bfloat16()), {}), ((q.double(), None), {}), ((None, None), {}), ((q, kk, kk[:, :1]), {}), ((q, None, kk), {}),
                     ((q, kk), dict(q_out=q[:3])), ((q, kk), dict(kv=kv)), ((q, kk), dict(chunk=c, kv=kv, k_out=kk)), ((q, None), dict(positions=i32(1, 2))),
                     ((q.requires_grad_(False).clone().requires_grad_(), None), dict(positions=i32(1, 2, 3, 4)))):
        with pytest.raises(ValueError):
            pkg.rope(p, *args, **kw)
    with pytest.raises(ValueError, match="GPU"):
        pkg.rope(p, q, kk, kk, chunk=c, kv=kv)
    for kw in (dict(out=q[:3]), dict(out=q.bfloat16()), dict(slopes=torch.zeros(3)), dict(prefix=i32(1)), dict(workspace=torch.zeros(9)), dict(prefix=torch.zeros(2))):
        with pytest.raises(ValueError):
            pkg.chunk_attention(q, kv, c, **kw)
    with pytest.raises(ValueError):
        pkg.chunk_attention(q[:3], kv, c)
    with pytest.raises(ValueError):
        pkg.chunk_attention(q, pkg.PagedKV(k, k, torch.zeros(3, 4, dtype=torch.int32)), c)
    with pytest.raises(pkg.EagleError):
        pkg.chunk_attention(q.bfloat16(), kv, c)                                # bf16 queries over an fp32 cache
    x = torch.zeros(R, 50)
    with pytest.raises(ValueError):
        pkg.LogitRules()
    with pytest.raises(ValueError):
        pkg.LogitRules(torch.zeros(2, 5, dtype=torch.int32))
    with pytest.raises(ValueError):
        pkg.LogitRules(torch.zeros(3, 5, dtype=torch.int32), i32(1, 2))
    with pytest.raises(ValueError):
        pkg.LogitRules(n_seqs=2, repetition=torch.zeros(3))
    with pytest.raises(ValueError):
        pkg.LogitRules(bias=(i32(0, 1, 2), i32(4, 5), torch.zeros(3)))
    r = pkg.LogitRules(n_seqs=2)
    for kw in (dict(row_start=i32(0, 2)), dict(path_token=i32(1, 2)), dict(allowed=torch.zeros(4, 1, dtype=torch.int32)), dict(allowed=torch.zeros(3, 2, dtype=torch.int32)), dict(out=x[:2])):
        with pytest.raises(ValueError):
            pkg.apply_logit_rules(x, r, **kw)
    with pytest.raises(ValueError):
        pkg.apply_logit_rules(x.double(), r)
    with pytest.raises(ValueError, match="GPU"):
        pkg.apply_logit_rules(x, r, row_start=i32(0, 2, 4))


def test_rows_that_lie_on_each_other():
    k = torch.zeros(9, 2, 32, 64)
    table = torch.zeros(1, 4, dtype=torch.int32)
    pkg.PagedKV(k, k, table)
    with pytest.raises(ValueError, match="page_table"):
        pkg.PagedKV(k, k, table.expand(3, 4))
    x, r = torch.zeros(4, 50), pkg.LogitRules(n_seqs=4)
    with pytest.raises(ValueError, match="allowed"):
        pkg.apply_logit_rules(x, r, allowed=torch.zeros(1, 2, dtype=torch.int32).expand(4, 2))


def test_the_most_tokens(lib):
    for r in (dict(max_tokens=-1), dict(max_tokens=2 ** 29 + 1)):
        call = ops.EagleLogits(n_rows=4, vocab=100, in_=A, out=A, in_stride=100, out_stride=100), ops.EagleLogitRules(n_seqs=4, tokens=A, n_tokens=A, token_stride=8, **r)
        assert lib.eagle_apply_logit_rules(*call, None) == EINVAL, r
    assert lib.eagle_apply_logit_rules(ops.EagleLogits(n_rows=1, vocab=2 ** 30 + 1, in_=A, out=A, in_stride=2 ** 31, out_stride=2 ** 31), ops.EagleLogitRules(n_seqs=1), None) == EINVAL


def test_outputs_that_lie_on_each_other_and_scores_out_of_range(lib):
    good = dict(n_rows=4, n_heads=4, dtype=0, q=A, q_out=A, q_row=256, q_head=64, q_out_row=256, q_out_head=64, positions=A)
    for bad in (dict(q_out_row=0), dict(q_out_head=0)):
        assert lib.eagle_rope(plan(), ops.EagleRopeArgs(**{**good, **bad}), None, None, None) == EINVAL, bad
    att = dict(n_heads=4, dtype=0, q=A, out=A, q_row=256, q_head=64, out_row=256, out_head=64, scale=0.1)
    size = lambda **kw: lib.eagle_chunk_attention_workspace(ops.EagleAttentionArgs(**{**att, **kw}), chunk(), paged())
    assert size() > 0 and size(softcap=1e-30) > 0
    for bad in (dict(out_row=0), dict(out_head=0), dict(softcap=1e-39), dict(scale=3e38), dict(scale=1e20, softcap=1e-20)):
        assert size(**bad) == 0, bad
    # bounds left wide need what tight ones need
    a = ops.EagleAttentionArgs(**att)
    assert lib.eagle_chunk_attention_workspace(a, chunk(max_rows=2 ** 30, max_keys=2 ** 30), paged()) == lib.eagle_chunk_attention_workspace(a, chunk(max_rows=4, max_keys=128), paged())
