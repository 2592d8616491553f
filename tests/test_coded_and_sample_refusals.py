"""What the operators over a cache of 8-bit codes and the choice of a token refuse, before anything is launched: at the C entry (no GPU needed: the addresses are never followed), in the binding,
and beside autograd."""
import ctypes

import pytest
import torch

import paper_2401_15077_amd as pkg
from paper_2401_15077_amd import operators as ops

A = 1 << 20                                                       # an address, never followed
EINVAL, ENOMEM = -1, -2
E4M3, INT8 = 2, 3


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2401_15077_amd import build
        build.build()
    return pkg.load_library()


def chunk(**kw):
    return ops.EagleChunk(**{**dict(n_seqs=2, n_rows=4, max_rows=3, max_keys=100, row_start=A, key_len=A), **kw})


def coded(**kw):
    return ops.EagleCodedKV(**{**dict(k=A, v=A, k_scale=A, v_scale=A, dtype=E4M3, n_kv_heads=2, head_dim=64, page_tokens=32, block_tokens=16, n_pages=9, pages_per_seq=4, page_stride=2 * 32 * 64,
                                      head_stride=32 * 64, token_stride=64, table_stride=4, scale_page=4, scale_head=2, page_table=A), **kw})


BAD_CHUNKS = [dict(n_seqs=0), dict(n_rows=-1), dict(max_rows=0), dict(max_keys=0), dict(row_start=None), dict(key_len=None), dict(tree_base=A), dict(tree_mask=A)]
BAD_CACHES = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(page_table=None), dict(dtype=0), dict(dtype=1), dict(dtype=4), dict(n_kv_heads=0), dict(page_tokens=0),
              dict(page_tokens=24), dict(page_tokens=8), dict(block_tokens=8), dict(block_tokens=24), dict(block_tokens=64), dict(block_tokens=0), dict(page_tokens=512, block_tokens=256), dict(n_pages=0),
              dict(pages_per_seq=0), dict(page_stride=0), dict(head_stride=-64), dict(token_stride=0), dict(table_stride=3), dict(scale_page=0), dict(scale_head=0), dict(k_scale=A + 2), dict(v_scale=A + 1)]


def test_append(lib):
    good = dict(n_rows=4, n_heads=4, n_kv_heads=2, dtype=1, q=A, k=A + (1 << 16), v=A + (2 << 16), q_out=A, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, q_out_row=256, q_out_head=64)

    def call(c=None, kv=None, p=None, **kw):
        return lib.eagle_rope_coded(pkg.rope_plan(64) if p is None else p, ops.EagleRopeArgs(**{**good, **kw}), c, kv, None)

    for kw in (dict(dtype=2), dict(n_rows=-1), dict(n_rows=5), dict(k=None), dict(q_out=None), dict(k_out=A), dict(inverse=1), dict(n_kv_heads=4), dict(n_heads=0), dict(q_out=A + 4),
               dict(q_out=A + (1 << 16), q_out_row=128)):
        assert call(chunk(), coded(), **kw) == EINVAL, kw
    assert call(chunk(), coded(head_dim=128)) == EINVAL and call(chunk(), None) == EINVAL and call(None, coded(), positions=A) == EINVAL
    assert call(chunk(), coded(), p=ops.EagleRopePlan()) == EINVAL
    assert lib.eagle_rope_coded(None, None, None, None, None) == EINVAL
    for bad in BAD_CHUNKS:
        assert call(chunk(**bad), coded()) == EINVAL, bad
    for bad in BAD_CACHES:
        assert call(chunk(), coded(**bad)) == EINVAL, bad
    assert call(chunk(n_rows=0), coded(), n_rows=0) == 0          # nothing to do
    # a cache of codes is none of the other entry's
    assert lib.eagle_rope(pkg.rope_plan(64), ops.EagleRopeArgs(**good), chunk(), ops.EaglePagedKV(k=A, v=A, dtype=E4M3, n_kv_heads=2, head_dim=64, page_tokens=32, n_pages=9, pages_per_seq=4,
                                                                                                 page_stride=4096, head_stride=2048, token_stride=64, table_stride=4, page_table=A), None) == EINVAL


def test_attention(lib):
    good = dict(n_heads=4, dtype=1, q=A, out=A, q_row=256, q_head=64, out_row=256, out_head=64, scale=0.1)

    def call(c=None, kv=None, ws=A, size=1 << 40, **kw):
        a, c, kv = ops.EagleAttentionArgs(**{**good, **kw}), c or chunk(), kv or coded()
        rc = lib.eagle_chunk_attention_coded(a, c, kv, ws, size, None)
        if ws == A and size == 1 << 40:
            assert (lib.eagle_chunk_attention_coded_workspace(a, c, kv) == 0) == (rc == EINVAL)
        return rc

    for kw in (dict(dtype=2), dict(n_heads=0), dict(n_heads=3), dict(q=None), dict(out=None), dict(scale=float("nan")), dict(softcap=-1.0), dict(softcap=float("inf")), dict(softcap=1e-39),
               dict(window=-1), dict(q=A + 8), dict(out=A + 8), dict(q_row=252), dict(q_head=60), dict(out_row=260), dict(out_head=68), dict(out_row=0), dict(out=A + 128)):
        assert call(**kw) == EINVAL, kw
    for kv in (dict(head_dim=144), dict(head_dim=72), dict(head_dim=8), dict(k=A + 8), dict(v=A + 4), dict(token_stride=72), dict(head_stride=2056), dict(page_stride=4104), dict(token_stride=2 ** 25)):
        assert call(kv=coded(**kv)) == EINVAL, kv
    for bad in BAD_CHUNKS:
        assert call(c=chunk(**bad)) == EINVAL, bad
    for bad in BAD_CACHES:
        assert call(kv=coded(**bad)) == EINVAL, bad
    assert call(ws=None) == EINVAL and call(ws=A + 64) == EINVAL
    for dtype in (E4M3, INT8):
        need = lib.eagle_chunk_attention_coded_workspace(ops.EagleAttentionArgs(**good), chunk(), coded(dtype=dtype))
        assert need > 0 and call(kv=coded(dtype=dtype), size=need - 1) == ENOMEM
    assert lib.eagle_chunk_attention_coded(None, None, None, None, 0, None) == EINVAL
    a = ops.EagleAttentionArgs(**good)                            # bounds left wide need what tight ones need
    assert lib.eagle_chunk_attention_coded_workspace(a, chunk(max_rows=2 ** 30, max_keys=2 ** 30), coded()) == lib.eagle_chunk_attention_coded_workspace(a, chunk(max_rows=4, max_keys=128), coded())


def test_sample(lib):
    good = dict(n_rows=4, vocab=100, dtype=0, logits=A, stride=100, uniform=A << 1, temperature=A << 2, top_k=A << 3, top_p=A << 4, min_p=A << 5, token=A << 6, logprob=A << 7)

    def call(ws=A << 8, size=1 << 30, **kw):
        a = ops.EagleSampleArgs(**{**good, **kw})
        rc = lib.eagle_sample(a, ws, size, None)
        if ws == A << 8 and size == 1 << 30:
            assert (lib.eagle_sample_workspace(a) == 0) == (rc == EINVAL)
        return rc

    for kw in (dict(dtype=2), dict(n_rows=-1), dict(n_rows=2 ** 24 + 1), dict(vocab=0), dict(vocab=2 ** 30 + 1), dict(logits=None), dict(uniform=None), dict(token=None), dict(stride=99), dict(logits=A + 2),
               dict(token=A + 4), dict(logprob=A + 1596), dict(token=A << 1), dict(logprob=(A << 4) + 12), dict(logprob=(A << 6) + 4), dict(token=(A << 6) + 2), dict(top_k=(A << 3) + 1),
               dict(token=(A << 3) - 12)):
        assert call(**kw) == EINVAL, kw
    assert call(ws=None) == EINVAL and call(ws=(A << 8) + 64) == EINVAL
    need = lib.eagle_sample_workspace(ops.EagleSampleArgs(**good))
    assert need > 0 and call(size=need - 1) == ENOMEM
    assert lib.eagle_sample(None, None, 0, None) == EINVAL and lib.eagle_sample_workspace(None) == 0
    assert call(n_rows=0) == 0                                    # nothing to do


# ----------------------------------------------------------------------------- the binding
R, S, H, KVH, D, V = 4, 2, 4, 2, 64, 50


def i32(*a):
    return torch.tensor(a, dtype=torch.int32)


def f32(*shape):
    return torch.zeros(*shape)


def codes(dtype=torch.int8):
    return torch.zeros(9, KVH, 32, D, dtype=torch.int8).view(dtype)


def cache(k=None, v=None, ks=None, vs=None, table=None):
    return pkg.PagedKV8(codes() if k is None else k, codes() if v is None else v, torch.zeros(S, 4, dtype=torch.int32) if table is None else table, f32(9, KVH, 2) if ks is None else ks,
                        f32(9, KVH, 2) if vs is None else vs)


def rows():
    return pkg.Chunk(i32(0, 2, 4), i32(5, 6), R, 2, 10)


def test_the_handle():
    assert cache().c.block_tokens == 16 and cache(codes(torch.float8_e4m3fn), codes(torch.float8_e4m3fn)).c.dtype == E4M3
    c = codes()
    for bad in ((c, c[:8]), (c, codes(torch.float8_e4m3fn)), (c.float(), c.float()), (c.view(torch.uint8), c.view(torch.uint8)), (c, c.transpose(1, 2).contiguous().transpose(1, 2)),
                (c[..., ::2], c[..., ::2])):
        with pytest.raises(ValueError, match="k and v|consecutive"):
            cache(*bad)
    s = f32(9, KVH, 2)
    for bad in ((s.double(), s), (s, s[:8]), (f32(9, KVH, 3), f32(9, KVH, 3)), (s, f32(9, KVH, 4)), (f32(9, KVH), s), (f32(9, KVH, 4)[..., ::2], f32(9, KVH, 4)[..., ::2]),
                (s, f32(KVH, 9, 2).transpose(0, 1)), (f32(9, KVH, 0), f32(9, KVH, 0))):
        with pytest.raises(ValueError, match="scale"):
            cache(ks=bad[0], vs=bad[1])
    for table in (torch.zeros(S, 4, dtype=torch.int64), torch.zeros(1, 4, dtype=torch.int32).expand(S, 4)):
        with pytest.raises(ValueError, match="page_table"):
            cache(table=table)


def test_calls_over_it():
    q, k, kv, c = f32(R, H, D), f32(R, KVH, D), cache(), rows()
    p = pkg.rope_plan(D)
    for args, kw in (((q, None), dict(chunk=c)), ((q, k), dict()), ((q, k), dict(chunk=c, k_out=k)), ((q, k[:3]), dict(chunk=c)), ((q, k, k[:, :1]), dict(chunk=c))):
        with pytest.raises((ValueError, pkg.EagleError)):
            pkg.rope(p, *args, kv=kv, **kw)
    with pytest.raises(ValueError, match="GPU"):
        pkg.rope(p, q, k, k, chunk=c, kv=kv)
    for kw in (dict(out=q[:3]), dict(out=q.bfloat16()), dict(slopes=f32(3)), dict(prefix=i32(1)), dict(workspace=f32(9))):
        with pytest.raises(ValueError):
            pkg.chunk_attention(q, kv, c, **kw)
    with pytest.raises(ValueError, match="sequences"):
        pkg.chunk_attention(q, cache(table=torch.zeros(3, 4, dtype=torch.int32)), c)
    with pytest.raises(pkg.EagleError, match="multiple of 16"):
        k8 = torch.zeros(9, KVH, 32, 72, dtype=torch.int8)
        pkg.chunk_attention(f32(R, H, 72), cache(k8, k8.clone()), c)
    with pytest.raises(pkg.EagleError, match="block_tokens"):
        pkg.chunk_attention(q, cache(ks=f32(9, KVH, 4), vs=f32(9, KVH, 4)), c)
    assert pkg.chunk_attention_workspace(q, kv, c) >= 256 and pkg.chunk_attention_workspace(q.bfloat16(), kv, c) >= 256


def test_sample_arguments():
    x, u = f32(R, V), f32(R)
    assert pkg.sample_workspace(x) >= 256 and pkg.sample_workspace(x.bfloat16()) >= 256
    for args, kw in (((x.double(), u), {}), ((x[0], u), {}), ((x[:, ::2], u), {}), ((x, u[:3]), {}), ((x, u.double()), {}), ((x, None), {}), ((x, u), dict(temperature=f32(3))),
                     ((x, u), dict(top_k=f32(R))), ((x, u), dict(top_p=i32(1, 2, 3, 4))), ((x, u), dict(min_p=f32(R, 1))), ((x, u), dict(token=f32(R))), ((x, u), dict(logprob=i32(1, 2, 3, 4))),
                     ((x, u), dict(workspace=f32(99)))):
        with pytest.raises(ValueError):
            pkg.sample(*args, **kw)
    with pytest.raises(ValueError, match="GPU"):
        pkg.sample(x, u)
    token, logprob = pkg.sample(x[:0], u[:0])
    assert token.shape == logprob.shape == (0,) and token.dtype == torch.int32


def leaf(*shape):
    return torch.zeros(*shape, requires_grad=True)


def attend(kv=None, **kw):
    return pkg.chunk_attention(kw.pop("q", f32(R, H, D)), kv or cache(), rows(), workspace=torch.zeros(1 << 20, dtype=torch.uint8), **kw)


def turn(kv=None, **kw):
    pkg.rope(pkg.rope_plan(D), kw.pop("q", f32(R, H, D)), kw.pop("k", f32(R, KVH, D)), kw.pop("v", f32(R, KVH, D)), chunk=rows(), kv=kv or cache(), **kw)


CALLS = {
    "k_scale, read": lambda t: attend(cache(ks=t(9, KVH, 2))), "v_scale, read": lambda t: attend(cache(vs=t(9, KVH, 2))), "k_scale, written": lambda t: turn(cache(ks=t(9, KVH, 2))),
    "v_scale, written": lambda t: turn(cache(vs=t(9, KVH, 2))), "q": lambda t: attend(q=t(R, H, D)), "out": lambda t: attend(out=t(R, H, D)), "slopes": lambda t: attend(slopes=t(H)),
    "k": lambda t: turn(k=t(R, KVH, D)), "v": lambda t: turn(v=t(R, KVH, D)), "q_out": lambda t: turn(q_out=t(R, H, D)),
    "logits": lambda t: pkg.sample(t(R, V), f32(R)), "uniform": lambda t: pkg.sample(f32(R, V), t(R)), "temperature": lambda t: pkg.sample(f32(R, V), f32(R), temperature=t(R)),
    "top_p": lambda t: pkg.sample(f32(R, V), f32(R), top_p=t(R)), "min_p": lambda t: pkg.sample(f32(R, V), f32(R), min_p=t(R)), "logprob": lambda t: pkg.sample(f32(R, V), f32(R), logprob=t(R)),
}


@pytest.mark.parametrize("name", CALLS)
def test_what_requires_gradients_is_refused(name, monkeypatch):
    monkeypatch.setattr(ops, "_call", lambda fn, device, *args: None)
    with pytest.raises(ValueError, match="requires gradients"):
        CALLS[name](leaf)
    CALLS[name](lambda *shape: leaf(*shape).detach())
    with torch.no_grad():
        CALLS[name](leaf)


def test_what_a_call_writes_counts_as_written(monkeypatch):
    monkeypatch.setattr(ops, "_call", lambda fn, device, *args: None)

    def versions(call, **named):
        before = {n: t._version for n, t in named.items()}
        call()
        return {n for n, t in named.items() if t._version != before[n]}

    q, k, v, q2, kc, vc, ks, vs, x, u, tok, lp = f32(R, H, D), f32(R, KVH, D), f32(R, KVH, D), f32(R, H, D), codes(), codes(), f32(9, KVH, 2), f32(9, KVH, 2), f32(R, V), f32(R), i32(0, 0, 0, 0), f32(R)
    every = dict(q=q, k=k, v=v, q2=q2, kc=kc, vc=vc, ks=ks, vs=vs, x=x, u=u, tok=tok, lp=lp)
    kv, c, plan = cache(kc, vc, ks, vs), rows(), pkg.rope_plan(D)
    assert versions(lambda: pkg.rope(plan, q, k, v, chunk=c, kv=kv), **every) == {"q", "kc", "vc", "ks", "vs"}
    assert versions(lambda: pkg.rope(plan, q, k, chunk=c, kv=kv, q_out=q2), **every) == {"q2", "kc", "ks"}
    assert versions(lambda: attend(kv, q=q, out=q2), **every) == {"q2"}
    assert versions(lambda: pkg.sample(x, u, token=tok, logprob=lp), **every) == {"tok", "lp"}


@pytest.mark.parametrize("first", ["pkg.load_library(need_gpu_runtime=False)", "pkg.load_library()", "None"])
def test_the_calls_are_declared(first):
    import os
    import subprocess
    import sys
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2401_15077_amd import build
        build.build()
    code = f"""
import ctypes
import paper_2401_15077_amd as pkg
import torch
first = {first}
from paper_2401_15077_amd import operators as ops
lib = ops._library()
for name in ("eagle_rope_coded", "eagle_chunk_attention_coded_workspace", "eagle_chunk_attention_coded", "eagle_sample_workspace", "eagle_sample"):
    assert getattr(lib, name).argtypes, name
assert lib.eagle_chunk_attention_coded_workspace.restype is lib.eagle_sample_workspace.restype is ctypes.c_size_t
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-1500:]
