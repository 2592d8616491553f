"""Operators on the caller's own tensors: rotary positions with the append to a paged cache, attention of a chunk of new tokens over it, both for caches of
8-bit codes too, the rules that logits pass before a token is chosen, and the choice (argument marshalling only; include/eagle.h has the definitions).

Every call is enqueued on torch's current stream of the tensors' device and does not synchronise.  Outputs are not recorded by autograd: tensors that
require gradients (inputs, outputs, slopes, and what a cache's or rules' handle was made from) are refused while gradients are enabled."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple, Union

import torch

from . import EAGLE_BF16, EAGLE_E4M3, EAGLE_F32, EAGLE_INT8, EagleError, load_library

_i32, _i64, _vp, _f32, _f64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_double
_TYPES = {torch.float32: EAGLE_F32, torch.bfloat16: EAGLE_BF16}
_CODES = {torch.float8_e4m3fn: EAGLE_E4M3, torch.int8: EAGLE_INT8}
ROPE_SCALINGS = ("none", "linear", "base", "bands", "ramp")


class EagleChunk(ctypes.Structure):
    _fields_ = [("n_seqs", _i32), ("n_rows", _i32), ("max_rows", _i32), ("max_keys", _i32), ("row_start", _vp), ("key_len", _vp), ("tree_base", _vp), ("tree_mask", _vp)]


class EaglePagedKV(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("dtype", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("page_tokens", _i32), ("n_pages", _i32), ("pages_per_seq", _i32),
                ("page_stride", _i64), ("head_stride", _i64), ("token_stride", _i64), ("table_stride", _i64), ("page_table", _vp)]


class EagleCodedKV(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("dtype", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("page_tokens", _i32), ("block_tokens", _i32),
                ("n_pages", _i32), ("pages_per_seq", _i32), ("page_stride", _i64), ("head_stride", _i64), ("token_stride", _i64), ("table_stride", _i64), ("scale_page", _i64),
                ("scale_head", _i64), ("page_table", _vp)]


class EagleRopeConfig(ctypes.Structure):
    _fields_ = [("head_dim", _i32), ("rot_dim", _i32), ("interleaved", _i32), ("scaling", _i32), ("theta", _f64), ("factor", _f64), ("low", _f64), ("high", _f64),
                ("trained_len", _i32), ("mscale", _f32)]


class EagleRopePlan(ctypes.Structure):
    _fields_ = [("head_dim", _i32), ("rot_dim", _i32), ("interleaved", _i32), ("mscale", _f32), ("turn", ctypes.c_uint64 * 128)]


class EagleRopeArgs(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("n_heads", _i32), ("n_kv_heads", _i32), ("dtype", _i32), ("inverse", _i32), ("q", _vp), ("k", _vp), ("v", _vp), ("q_out", _vp), ("k_out", _vp),
                ("q_row", _i64), ("q_head", _i64), ("k_row", _i64), ("k_head", _i64), ("v_row", _i64), ("v_head", _i64), ("q_out_row", _i64), ("q_out_head", _i64),
                ("k_out_row", _i64), ("k_out_head", _i64), ("positions", _vp)]


class EagleAttentionArgs(ctypes.Structure):
    _fields_ = [("n_heads", _i32), ("dtype", _i32), ("window", _i32), ("q", _vp), ("out", _vp), ("q_row", _i64), ("q_head", _i64), ("out_row", _i64), ("out_head", _i64),
                ("scale", _f32), ("softcap", _f32), ("slopes", _vp), ("prefix", _vp)]


class EagleLogitRules(ctypes.Structure):
    _fields_ = [("n_seqs", _i32), ("tokens", _vp), ("token_stride", _i64), ("max_tokens", _i32), ("n_tokens", _vp), ("n_prompt", _vp), ("repetition", _vp), ("presence", _vp), ("frequency", _vp),
                ("bias_start", _vp), ("bias_token", _vp), ("bias_value", _vp), ("n_bias", _i32)]


class EagleLogits(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("vocab", _i32), ("dtype", _i32), ("n_masks", _i32), ("in_", _vp), ("out", _vp), ("in_stride", _i64), ("out_stride", _i64), ("mask_stride", _i64),
                ("row_start", _vp), ("path_token", _vp), ("path_mask", _vp), ("allowed", _vp), ("allowed_row", _vp)]


class EagleSampleArgs(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("vocab", _i32), ("dtype", _i32), ("logits", _vp), ("stride", _i64), ("uniform", _vp), ("temperature", _vp), ("top_k", _vp), ("top_p", _vp), ("min_p", _vp),
                ("token", _vp), ("logprob", _vp)]


class EagleAttentionRules(ctypes.Structure):
    _fields_ = [("softcap", _f32), ("window", _i32), ("slopes_dev", _vp)]


class EagleContextRules(ctypes.Structure):
    _fields_ = [("repetition", _vp), ("presence", _vp), ("frequency", _vp), ("bias_start", _vp), ("bias_token", _vp), ("bias_value", _vp), ("n_bias", _i32), ("n_masks", _i32),
                ("allowed", _vp), ("mask_stride", _i64), ("allowed_row", _vp)]


def declare(lib) -> None:
    """Argument types of the entry points."""
    P = ctypes.POINTER
    lib.eagle_rope_plan_init.argtypes = [P(EagleRopeConfig), P(EagleRopePlan)]
    lib.eagle_rope.argtypes = [P(EagleRopePlan), P(EagleRopeArgs), P(EagleChunk), P(EaglePagedKV), _vp]
    lib.eagle_chunk_attention_workspace.argtypes = [P(EagleAttentionArgs), P(EagleChunk), P(EaglePagedKV)]
    lib.eagle_chunk_attention_workspace.restype = ctypes.c_size_t
    lib.eagle_chunk_attention.argtypes = [P(EagleAttentionArgs), P(EagleChunk), P(EaglePagedKV), _vp, ctypes.c_size_t, _vp]
    lib.eagle_rope_coded.argtypes = [P(EagleRopePlan), P(EagleRopeArgs), P(EagleChunk), P(EagleCodedKV), _vp]
    lib.eagle_chunk_attention_coded_workspace.argtypes = [P(EagleAttentionArgs), P(EagleChunk), P(EagleCodedKV)]
    lib.eagle_chunk_attention_coded_workspace.restype = ctypes.c_size_t
    lib.eagle_chunk_attention_coded.argtypes = [P(EagleAttentionArgs), P(EagleChunk), P(EagleCodedKV), _vp, ctypes.c_size_t, _vp]
    lib.eagle_sample_workspace.argtypes = [P(EagleSampleArgs)]
    lib.eagle_sample_workspace.restype = ctypes.c_size_t
    lib.eagle_sample.argtypes = [P(EagleSampleArgs), _vp, ctypes.c_size_t, _vp]
    lib.eagle_set_rope.argtypes = [_vp, P(EagleRopeConfig)]
    lib.eagle_set_attention.argtypes = [_vp, P(EagleAttentionRules)]
    lib.eagle_set_logit_rules.argtypes = [_vp, P(EagleContextRules)]
    lib.eagle_apply_logit_rules.argtypes = [P(EagleLogits), P(EagleLogitRules), _vp]


# tells autograd that tensors it may have saved are no longer what they were
_written = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device      # (a tensor on the device: the runtime is up)
_lib = None


def _library():
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


def _call(fn, device, *args):
    """Calls fn(*args, stream) with the tensors' device current."""
    if device.type != "cuda":
        raise ValueError(f"the tensors are on {device}: libeagle needs a GPU (no CPU fallback exists)")
    index = device.index
    if _current_device() != index:
        with torch.cuda.device(index):
            rc = fn(*args, _raw_stream(index))
    else:
        rc = fn(*args, _raw_stream(index))
    if rc != 0:
        raise EagleError(rc, _library().eagle_last_error().decode())


def _plain(t: torch.Tensor, name: str) -> None:
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires gradients: libeagle's operators are not recorded by autograd")


def _list(t: Optional[torch.Tensor], name: str, dtype, n: Optional[int], device) -> Optional[int]:
    """Address of a contiguous 1-D tensor of n entries (None: any number) on `device`; None for None."""
    if t is None:
        return None
    if t.dtype != dtype or t.dim() != 1 or (n is not None and t.shape[0] != n) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {'any number of' if n is None else n} entries on {device}: got {t.dtype} {tuple(t.shape)} on {t.device}")
    if t.requires_grad:
        _plain(t, name)
    return t.data_ptr()


def _heads(t: torch.Tensor, name: str, rows: Optional[int], heads: Optional[int], dim: int, dtype=None, device=None):
    """Address, row stride and head stride of a [rows, heads, head_dim] tensor (None: any number)."""
    shape = t.shape
    if len(shape) != 3 or shape[2] != dim or (rows is not None and shape[0] != rows) or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must be [rows, heads, head_dim] = {[rows, heads, dim]}: got {list(shape)}")
    if dtype is None:
        if t.dtype not in _TYPES:
            raise ValueError(f"{name} must be float32 or bfloat16: got {t.dtype}")
    elif t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} on {device}: got {t.dtype} on {t.device}")
    stride = t.stride()
    if stride[2] != 1 and dim > 1:
        raise ValueError(f"the elements of a head of {name} must be consecutive")
    if t.requires_grad:
        _plain(t, name)
    return t.data_ptr(), stride[0], stride[1]


def _masks(allowed: torch.Tensor, vocab: int, device):
    """Address, number and row stride (in words) of the masks `allowed`."""
    if allowed.dtype != torch.int32 or allowed.dim() != 2 or allowed.device != device or (allowed.stride(1) != 1 and allowed.shape[1] > 1) or allowed.shape[1] * 32 < vocab \
            or (allowed.shape[0] > 1 and allowed.stride(0) < allowed.shape[1]):
        raise ValueError(f"allowed must be an int32 [masks, words] tensor on {device} of at least {(vocab + 31) // 32} consecutive words a row, its rows apart")
    return allowed.data_ptr(), allowed.shape[0], max(allowed.stride(0), allowed.shape[1])


class Chunk:
    """New tokens of a batch: int32 row_start [n_seqs + 1], key_len [n_seqs]; for draft trees int32 tree_base [n_seqs] and int64 tree_mask [n_rows].
    max_rows / max_keys bound the rows of a sequence and key_len."""

    def __init__(self, row_start: torch.Tensor, key_len: torch.Tensor, n_rows: int, max_rows: int, max_keys: int, *, tree_base: Optional[torch.Tensor] = None,
                 tree_mask: Optional[torch.Tensor] = None):
        self.device, self.n_seqs, self.n_rows = key_len.device, key_len.shape[0], int(n_rows)
        self._keep = (row_start, key_len, tree_base, tree_mask)
        self.c = EagleChunk(self.n_seqs, self.n_rows, int(max_rows), int(max_keys), _list(row_start, "row_start", torch.int32, self.n_seqs + 1, self.device),
                            _list(key_len, "key_len", torch.int32, self.n_seqs, self.device), _list(tree_base, "tree_base", torch.int32, self.n_seqs, self.device),
                            _list(tree_mask, "tree_mask", torch.int64, self.n_rows, self.device))


def _page_table(page_table: torch.Tensor, device) -> None:
    if page_table.dtype != torch.int32 or page_table.dim() != 2 or page_table.device != device or (page_table.stride(1) != 1 and page_table.shape[1] > 1) \
            or (page_table.shape[0] > 1 and page_table.stride(0) < page_table.shape[1]):
        raise ValueError(f"page_table must be an int32 [n_seqs, pages] tensor on {device}, its rows consecutive and apart")


class PagedKV:
    """A paged cache: k, v [n_pages, n_kv_heads, page_tokens, head_dim] of the same type and strides, int32 page_table [n_seqs, pages]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride() or k.device != v.device or k.dtype not in _TYPES:
            raise ValueError("k and v must be [n_pages, n_kv_heads, page_tokens, head_dim], float32 or bfloat16, of the same type, shape and strides on one device")
        if k.stride(3) != 1 and k.shape[3] > 1:
            raise ValueError("the elements of a token of k and v must be consecutive")
        _page_table(page_table, k.device)
        self.device, self.dtype, self.n_seqs, self.n_kv_heads, self.head_dim = k.device, k.dtype, page_table.shape[0], k.shape[1], k.shape[3]
        self.both, self._table, self.grads = (k, v), page_table, k.requires_grad or v.requires_grad
        self.of_k = (k,)                                          # what an append of keys alone writes
        self.c = EaglePagedKV(k.data_ptr(), v.data_ptr(), _TYPES[k.dtype], k.shape[1], k.shape[3], k.shape[2], k.shape[0], page_table.shape[1], k.stride(0), k.stride(1), k.stride(2),
                              max(page_table.stride(0), page_table.shape[1]), page_table.data_ptr())


class PagedKV8:
    """A paged cache of 8-bit codes: k, v [n_pages, n_kv_heads, page_tokens, head_dim], float8_e4m3fn or int8, of the same type and strides, with float32 k_scale, v_scale [n_pages, n_kv_heads,
    blocks] of the same strides, a scale for each page_tokens / blocks tokens; int32 page_table [n_seqs, pages].  An element is code * scale."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride() or k.device != v.device or k.dtype not in _CODES:
            raise ValueError("k and v must be [n_pages, n_kv_heads, page_tokens, head_dim], float8_e4m3fn or int8, of the same type, shape and strides on one device")
        if k.stride(3) != 1 and k.shape[3] > 1:
            raise ValueError("the elements of a token of k and v must be consecutive")
        _page_table(page_table, k.device)
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.dtype != torch.float32 or t.device != k.device or t.dim() != 3 or t.shape[:2] != k.shape[:2] or t.shape[2] < 1 or k.shape[2] % t.shape[2] or t.shape != k_scale.shape \
                    or t.stride() != k_scale.stride() or (t.stride(2) != 1 and t.shape[2] > 1):
                raise ValueError(f"{name} must be a float32 [n_pages, n_kv_heads, blocks of a page] tensor on {k.device}, a page's scales of a head consecutive, both of the same shape and strides")
        self.device, self.dtype, self.n_seqs, self.n_kv_heads, self.head_dim = k.device, k.dtype, page_table.shape[0], k.shape[1], k.shape[3]
        self.both, self._table = (k, v, k_scale, v_scale), page_table
        self.grads = any(t.requires_grad for t in self.both)
        self.of_k = (k, k_scale)
        self.c = EagleCodedKV(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), _CODES[k.dtype], k.shape[1], k.shape[3], k.shape[2], k.shape[2] // k_scale.shape[2], k.shape[0],
                              page_table.shape[1], k.stride(0), k.stride(1), k.stride(2), max(page_table.stride(0), page_table.shape[1]), k_scale.stride(0), k_scale.stride(1),
                              page_table.data_ptr())


def _same_batch(chunk: Chunk, kv: PagedKV, device) -> None:
    if chunk.device != device or kv.device != device:
        raise ValueError(f"the chunk is on {chunk.device}, the cache on {kv.device}, the rows on {device}")
    if kv.n_seqs != chunk.n_seqs:
        raise ValueError(f"the page table has {kv.n_seqs} sequences, the chunk {chunk.n_seqs}")
    if kv.grads:
        for t, name in zip(kv.both, ("k of the cache", "v of the cache", "k_scale", "v_scale")):
            _plain(t, name)


def rope_config(head_dim: int, *, theta: float = 10000.0, rot_dim: Optional[int] = None, interleaved: bool = False, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                high: float = 4.0, trained_len: int = 4096, mscale: float = 1.0) -> EagleRopeConfig:
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {ROPE_SCALINGS}: got {scaling!r}")
    return EagleRopeConfig(head_dim, head_dim if rot_dim is None else rot_dim, int(interleaved), ROPE_SCALINGS.index(scaling), theta, factor, low, high, trained_len, mscale)


def rope_plan(head_dim: int, *, theta: float = 10000.0, rot_dim: Optional[int] = None, interleaved: bool = False, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
              high: float = 4.0, trained_len: int = 4096, mscale: float = 1.0) -> EagleRopePlan:
    """How positions turn a head (see eagle_rope_config); scaling is one of ROPE_SCALINGS.  Host work: make it once."""
    lib = _library()
    cfg = rope_config(head_dim, theta=theta, rot_dim=rot_dim, interleaved=interleaved, scaling=scaling, factor=factor, low=low, high=high, trained_len=trained_len, mscale=mscale)
    plan = EagleRopePlan()
    rc = lib.eagle_rope_plan_init(ctypes.byref(cfg), ctypes.byref(plan))
    if rc != 0:
        raise EagleError(rc, lib.eagle_last_error().decode())
    return plan


def rope(plan: EagleRopePlan, q: Optional[torch.Tensor], k: Optional[torch.Tensor], v: Optional[torch.Tensor] = None, *, chunk: Optional[Chunk] = None,
         kv: Union[PagedKV, PagedKV8, None] = None, positions: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
         inverse: bool = False) -> None:
    """Rotates q [rows, heads, head_dim] into q_out (None: in place) and k [rows, kv heads, head_dim] into the cache `kv`, with v, or without a cache into
    k_out (None: in place).  Over a PagedKV8 keys and values are rounded to codes of their blocks' scales (eagle_rope_coded)."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("neither q nor k is given")
    R, dtype, device, D = x.shape[0], x.dtype, x.device, plan.head_dim
    none = (None, 0, 0)
    qa = qo = ka = ko = va = none
    H = KVH = 0
    if q is not None:
        H = q.shape[1] if q.dim() > 1 else 0
        qa = _heads(q, "q", None, None, D)
        qo = qa if q_out is None else _heads(q_out, "q_out", R, H, D, dtype, device)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if k is not None:
        KVH = k.shape[1] if k.dim() > 1 else 0
        ka = _heads(k, "k", R, None, D, dtype, device) if q is not None else _heads(k, "k", None, None, D)
        if kv is None:
            ko = ka if k_out is None else _heads(k_out, "k_out", R, KVH, D, dtype, device)
        elif k_out is not None:
            raise ValueError("with a cache k goes there: k_out must be None")
        if v is not None:
            va = _heads(v, "v", R, KVH, D, dtype, device)
    elif k_out is not None or v is not None:
        raise ValueError("k_out or v without k")
    at = _list(positions, "positions", torch.int32, R, device)
    if kv is not None:
        if chunk is None:
            raise ValueError("a cache needs a chunk")
        _same_batch(chunk, kv, device)
    elif chunk is not None and chunk.device != device:
        raise ValueError(f"the chunk is on {chunk.device}, the rows on {device}")
    if R == 0:
        return
    a = EagleRopeArgs(R, H, KVH, _TYPES[dtype], int(inverse), qa[0], ka[0], va[0], qo[0], ko[0], qa[1], qa[2], ka[1], ka[2], va[1], va[2], qo[1], qo[2], ko[1], ko[2], at)
    lib = _library()
    _call(lib.eagle_rope_coded if type(kv) is PagedKV8 else lib.eagle_rope, device, plan, a, chunk.c if chunk is not None else None, kv.c if kv is not None else None)
    if q is not None:
        _written((q if q_out is None else q_out,))
    if k is not None:
        _written((k if k_out is None else k_out,) if kv is None else kv.both if v is not None else kv.of_k)


def _attention_args(q, kv, chunk, scale, softcap, slopes, window, prefix, out):
    D, device = kv.head_dim, q.device
    qa = _heads(q, "q", chunk.n_rows, None, D)
    H = q.shape[1]
    oa = qa if out is None else _heads(out, "out", chunk.n_rows, H, D, q.dtype, device)
    _same_batch(chunk, kv, device)
    return EagleAttentionArgs(H, _TYPES[q.dtype], window, qa[0], oa[0], qa[1], qa[2], oa[1], oa[2], D ** -0.5 if scale is None else scale, softcap,
                              _list(slopes, "slopes", torch.float32, H, device), _list(prefix, "prefix", torch.int32, chunk.n_seqs, device))


def _attention_calls(lib, kv):
    if type(kv) is PagedKV8:
        return lib.eagle_chunk_attention_coded_workspace, lib.eagle_chunk_attention_coded
    return lib.eagle_chunk_attention_workspace, lib.eagle_chunk_attention


def chunk_attention_workspace(q: torch.Tensor, kv: Union[PagedKV, PagedKV8], chunk: Chunk) -> int:
    """Bytes of workspace chunk_attention needs for these arguments (whatever the masks)."""
    lib = _library()
    a = _attention_args(q, kv, chunk, None, 0.0, None, 0, None, None)
    n = _attention_calls(lib, kv)[0](a, chunk.c, kv.c)
    if n == 0:
        raise EagleError(-1, lib.eagle_last_error().decode())
    return n


def chunk_attention(q: torch.Tensor, kv: Union[PagedKV, PagedKV8], chunk: Chunk, *, scale: Optional[float] = None, softcap: float = 0.0, slopes: Optional[torch.Tensor] = None, window: int = 0,
                    prefix: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(score) v of every row of q [rows, heads, head_dim] over the visible tokens of `kv` -> out (None: a new tensor).  scale: None = head_dim ** -0.5.
    workspace: a uint8 tensor of chunk_attention_workspace() bytes (None: one from torch's allocator for this call)."""
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    a = _attention_args(q, kv, chunk, scale, softcap, slopes, window, prefix, out)
    lib = _library()
    if chunk.n_rows == 0:
        return out
    size_of, attend = _attention_calls(lib, kv)
    if workspace is None:
        n = size_of(a, chunk.c, kv.c)
        if n == 0:
            raise EagleError(-1, lib.eagle_last_error().decode())
        workspace = torch.empty(n, dtype=torch.uint8, device=q.device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != q.device:
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {q.device}")
    _call(attend, q.device, a, chunk.c, kv.c, workspace.data_ptr(), workspace.numel())
    _written((out,))
    return out


class LogitRules:
    """Rules of a batch of sequences: int32 tokens [n_seqs, longest] with n_tokens [n_seqs] of them each, the first n_prompt [n_seqs] (None: 0) of which only
    `repetition` counts; float32 repetition, presence, frequency [n_seqs]; bias = (int32 start [n_seqs + 1], int32 token [n], float32 value [n])."""

    def __init__(self, tokens: Optional[torch.Tensor] = None, n_tokens: Optional[torch.Tensor] = None, *, n_seqs: Optional[int] = None, n_prompt: Optional[torch.Tensor] = None,
                 repetition: Optional[torch.Tensor] = None, presence: Optional[torch.Tensor] = None, frequency: Optional[torch.Tensor] = None,
                 bias: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None):
        given = [t for t in (n_tokens, n_prompt, repetition, presence, frequency) if t is not None]
        if bias is not None:
            given.append(bias[0])
        if not given and n_seqs is None:
            raise ValueError("without any rule n_seqs is needed")
        if (tokens is None) != (n_tokens is None):
            raise ValueError("tokens and n_tokens belong together")
        self.device = given[0].device if given else None
        S = n_seqs if n_seqs is not None else given[0].shape[0] - (given[0] is (bias[0] if bias is not None else None))
        if tokens is not None and (tokens.dtype != torch.int32 or tokens.dim() != 2 or tokens.shape[0] != S or tokens.device != self.device or (tokens.stride(1) != 1 and tokens.shape[1] > 1)):
            raise ValueError(f"tokens must be an int32 [{S}, longest] tensor on {self.device}, its rows consecutive")
        self.n_seqs, dev = int(S), self.device
        b = bias if bias is not None else (None, None, None)
        if bias is not None and b[1].shape != b[2].shape:
            raise ValueError("bias tokens and values must be equally many")
        self._keep = (tokens, n_tokens, n_prompt, repetition, presence, frequency, b)
        self.grads = [(t, name) for t, name in ((repetition, "repetition"), (presence, "presence"), (frequency, "frequency"), (b[2], "bias value")) if t is not None and t.requires_grad]
        self.longest = tokens.shape[1] if tokens is not None else 0
        f, i = torch.float32, torch.int32
        self.c = EagleLogitRules(self.n_seqs, tokens.data_ptr() if tokens is not None else None, tokens.stride(0) if tokens is not None else 0, self.longest,
                                 _list(n_tokens, "n_tokens", i, S, dev), _list(n_prompt, "n_prompt", i, S, dev), _list(repetition, "repetition", f, S, dev),
                                 _list(presence, "presence", f, S, dev), _list(frequency, "frequency", f, S, dev), _list(b[0], "bias start", i, S + 1, dev),
                                 _list(b[1], "bias token", i, None, dev), _list(b[2], "bias value", f, None, dev), b[1].shape[0] if bias is not None else 0)


def apply_logit_rules(logits: torch.Tensor, rules: LogitRules, *, row_start: Optional[torch.Tensor] = None, path_token: Optional[torch.Tensor] = None,
                      path_mask: Optional[torch.Tensor] = None, allowed: Optional[torch.Tensor] = None, allowed_row: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The rules on logits [rows, vocab] (float32 or bfloat16) -> out (None: in place).  row_start: int32 [n_seqs + 1] (None: one row a sequence).  path_token int32, path_mask int64
    [rows]: tokens along a draft tree.  allowed: int32 [masks, words >= vocab / 32], a bit a token; allowed_row: int32 [rows], the row's mask (-1: none; None: row r's is mask r)."""
    if logits.dim() != 2 or logits.dtype not in _TYPES or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be a float32 or bfloat16 [rows, vocab] tensor, its rows consecutive")
    if logits.requires_grad:
        _plain(logits, "logits")
    for t, name in rules.grads:                                   # (where they were made while gradients were off)
        _plain(t, name)
    R, V = logits.shape
    dev = logits.device
    if rules.device is not None and rules.device != dev:
        raise ValueError(f"the rules are on {rules.device}, the logits on {dev}")
    if out is None:
        out = logits
    elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != dev or (out.stride(1) != 1 and V > 1):
        raise ValueError(f"out must be {logits.dtype} {list(logits.shape)} on {dev}, its rows consecutive")
    elif out.requires_grad:
        _plain(out, "out")
    masks = (None, 0, 0)
    if allowed is not None:
        masks = _masks(allowed, V, dev)
        if allowed_row is None and allowed.shape[0] != R:
            raise ValueError(f"without allowed_row there is one mask a row ({allowed.shape[0]} masks, {R} rows)")
    l = EagleLogits(R, V, _TYPES[logits.dtype], masks[1], logits.data_ptr(), out.data_ptr(), logits.stride(0) if R > 1 else V, out.stride(0) if R > 1 else V, masks[2],
                    _list(row_start, "row_start", torch.int32, rules.n_seqs + 1, dev), _list(path_token, "path_token", torch.int32, R, dev),
                    _list(path_mask, "path_mask", torch.int64, R, dev), masks[0], _list(allowed_row, "allowed_row", torch.int32, R, dev))
    if R > 0:
        _call(_library().eagle_apply_logit_rules, dev, l, rules.c)
        _written((out,))
    return out


def _sample_args(logits, uniform, temperature, top_k, top_p, min_p, token, logprob):
    if logits.dim() != 2 or logits.dtype not in _TYPES or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be a float32 or bfloat16 [rows, vocab] tensor, its rows consecutive")
    if logits.requires_grad:
        _plain(logits, "logits")
    (R, V), dev, f = logits.shape, logits.device, torch.float32
    return EagleSampleArgs(R, V, _TYPES[logits.dtype], logits.data_ptr(), logits.stride(0) if R > 1 else V, _list(uniform, "uniform", f, R, dev), _list(temperature, "temperature", f, R, dev),
                           _list(top_k, "top_k", torch.int32, R, dev), _list(top_p, "top_p", f, R, dev), _list(min_p, "min_p", f, R, dev), _list(token, "token", torch.int32, R, dev),
                           _list(logprob, "logprob", f, R, dev))


def sample_workspace(logits: torch.Tensor) -> int:
    """Bytes of workspace sample needs for logits of this shape and type (whatever the filters)."""
    lib = _library()
    a = _sample_args(logits, None, None, None, None, None, None, None)
    a.logits, a.uniform, a.token = 1 << 60, 1 << 58, 1 << 56      # (sizes alone count here)
    n = lib.eagle_sample_workspace(a)
    if n == 0:
        raise EagleError(-1, lib.eagle_last_error().decode())
    return n


def sample(logits: torch.Tensor, uniform: torch.Tensor, *, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
           min_p: Optional[torch.Tensor] = None, token: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """A token of every row of logits [rows, vocab] (float32 or bfloat16), drawn by the row's number of float32 uniform [rows] in [0, 1) -> (int32 token [rows], float32 logprob [rows]), new
    tensors where none are given.  float32 temperature, top_p, min_p and int32 top_k [rows] (None: no such filter): see eagle_sample.
    workspace: a uint8 tensor of sample_workspace() bytes (None: one from torch's allocator for this call)."""
    if uniform is None:
        raise ValueError("uniform is needed: a random number for every row")
    if logits.dim() != 2:
        raise ValueError("logits must be a float32 or bfloat16 [rows, vocab] tensor, its rows consecutive")
    R, dev = logits.shape[0], logits.device
    if token is None:
        token = torch.empty(R, dtype=torch.int32, device=dev)
    if logprob is None:
        logprob = torch.empty(R, dtype=torch.float32, device=dev)
    a = _sample_args(logits, uniform, temperature, top_k, top_p, min_p, token, logprob)
    if R == 0:
        return token, logprob
    lib = _library()
    if workspace is None:
        n = lib.eagle_sample_workspace(a)
        if n == 0:
            raise EagleError(-1, lib.eagle_last_error().decode())
        workspace = torch.empty(n, dtype=torch.uint8, device=dev)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != dev:
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {dev}")
    _call(lib.eagle_sample, dev, a, workspace.data_ptr(), workspace.numel())
    _written((token, logprob))
    return token, logprob
