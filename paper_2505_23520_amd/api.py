"""Thin ctypes binding over libanchor_attention.so (see include/anchor_attention.h).

Argument marshalling only: every step of the path runs in the HIP kernels.
torch supplies device memory and the stream.  Importing this module fails if
the library has not been built (run ``python -m paper_2505_23520_amd.build``
or ``__graft_entry__.build()``); there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libanchor_attention.so")

AA_FP32, AA_BF16 = 0, 1
AA_STRIPE, AA_BLOCK = 0, 1
AA_KV_PLAIN, AA_KV_FP4 = 0, 1
AA_ENGINE_AUTO, AA_ENGINE_128, AA_ENGINE_256 = 0, 1, 2
AA_OK, AA_EINVAL, AA_EUNSUPPORTED, AA_EWORKSPACE, AA_EHIP = 0, -1, -2, -3, -4


class aa_params(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
        ("N", ctypes.c_int32), ("d", ctypes.c_int32),
        ("block_q", ctypes.c_int32), ("block_kv", ctypes.c_int32),
        ("n_init", ctypes.c_int32), ("window", ctypes.c_int32), ("step", ctypes.c_int32),
        ("theta", ctypes.c_float), ("softmax_scale", ctypes.c_float),
        ("causal", ctypes.c_int32), ("dtype", ctypes.c_int32), ("use_anchor", ctypes.c_int32),
        ("granularity", ctypes.c_int32), ("engine", ctypes.c_int32),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3),
        ("cu_seqlens", ctypes.c_void_p), ("total_tokens", ctypes.c_int64),
    ]


class aa_sizes(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("acc_elems", ctypes.c_int64), ("blk_cap", ctypes.c_int64),
        ("blocks", ctypes.c_int64), ("grp_cap", ctypes.c_int64), ("groups", ctypes.c_int64),
        ("idx_capacity_max", ctypes.c_int64),
        ("select_ws_bytes", ctypes.c_size_t), ("prefill_ws_bytes", ctypes.c_size_t),
    ]


class aa_kv_params(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("N", ctypes.c_int32),
        ("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("format", ctypes.c_int32),
        ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32),
        ("max_len", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("rot_dim", ctypes.c_int32), ("rot_interleaved", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
        ("o_stride", ctypes.c_int64 * 3), ("ko_stride", ctypes.c_int64 * 3),
        ("kc", ctypes.c_void_p), ("vc", ctypes.c_void_p),
        ("kc_stride", ctypes.c_int64 * 3), ("vc_stride", ctypes.c_int64 * 3),
        ("ks", ctypes.c_void_p), ("vs", ctypes.c_void_p),
        ("ks_stride", ctypes.c_int64 * 3), ("vs_stride", ctypes.c_int64 * 3),
        ("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
        ("kv_len", ctypes.c_void_p), ("cu_seqlens", ctypes.c_void_p), ("total_tokens", ctypes.c_int64),
    ]


_P = ctypes.c_void_p
_PP = ctypes.POINTER(aa_params)
_PK = ctypes.POINTER(aa_kv_params)
_SIGNATURES = {
    "anchor_sizes": (ctypes.c_int, [_PP, ctypes.POINTER(aa_sizes)]),
    "anchor_workspace_bytes": (ctypes.c_int, [_PP, ctypes.POINTER(ctypes.c_size_t)]),
    "anchor_compute": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, _P, _P]),
    "stripe_select": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, ctypes.c_int64, _P, _P, ctypes.c_size_t, _P]),
    "stripe_select_noalloc": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, ctypes.c_int64, _P, _P]),
    "sparse_attn": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_int64, _P, _P, _P]),
    "anchor_attention_prefill": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "dense_causal_flash": (ctypes.c_int, [_PP, _P, _P, _P, _P, _P, _P]),
    "kv_append": (ctypes.c_int, [_PK, _P, _P, _P, _P, _P, _P, _P, _P]),
    "kv_attn_workspace_bytes": (ctypes.c_int, [_PK, ctypes.POINTER(ctypes.c_size_t)]),
    "kv_attn": (ctypes.c_int, [_PK, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "kv_read": (ctypes.c_int, [_PK, _P, _P, _P]),
    "anchor_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "anchor_last_hip_error": (ctypes.c_char_p, []),
}
EXPORTS = tuple(_SIGNATURES)


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """dlopen the built library and declare its signatures; ImportError if it is not there."""
    if not os.path.exists(path):
        raise ImportError(
            "libanchor_attention.so is not built (%s). Build it with "
            "`python -m paper_2505_23520_amd.build`; there is no fallback path." % path)
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


_lib = load_library()


class AnchorError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        msg = _lib.anchor_strerror(code).decode()
        if code == AA_EHIP:
            msg += ": " + _lib.anchor_last_hip_error().decode()
        super().__init__("anchor_attention error %d (%s)" % (code, msg))


def _check(rc: int):
    if rc != AA_OK:
        raise AnchorError(rc)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


@dataclass
class Config:
    """Method parameters (Algorithms 1-3 REQUIRE lines), token units."""
    block: int = 128
    n_init: int = 128
    window: int = 128
    step: int = 16
    theta: float = 12.0
    softmax_scale: float = 0.0
    use_anchor: bool = True
    causal: bool = True
    granularity: int = AA_STRIPE     # AA_BLOCK: one decision per key block (Sec. 2.1.2, Table 1)
    engine: int = AA_ENGINE_AUTO     # testing / tuning aid: force one of the two bf16 tile engines


def _strides(t: torch.Tensor, packed: bool):
    if packed:       # [H, total, d]
        assert t.dim() == 3 and t.stride(2) == 1
        return (0, t.stride(0), t.stride(1))
    assert t.dim() == 4 and t.stride(3) == 1   # [B, H, N, d]
    return (t.stride(0), t.stride(1), t.stride(2))


def make_params(cfg: Config, q, k, v, out=None, cu_seqlens=None, max_seqlen=None, total_tokens=None) -> aa_params:
    """Describe tensors q [B,Hq,N,d] / k,v [B,Hkv,N,d] (any strides with d contiguous), or,
    with cu_seqlens (device int32 [B+1]), packed q [Hq,total,d] / k,v [Hkv,total,d]."""
    packed = cu_seqlens is not None
    p = aa_params()
    if packed:
        p.B = cu_seqlens.numel() - 1
        p.Hq, p.Hkv, p.d = q.shape[0], k.shape[0], q.shape[2]
        p.N = int(max_seqlen)
        p.total_tokens = int(q.shape[1] if total_tokens is None else total_tokens)
        p.cu_seqlens = cu_seqlens.data_ptr()
    else:
        p.B, p.Hq, p.N, p.d = q.shape
        p.Hkv = k.shape[1]
        p.cu_seqlens = None
        p.total_tokens = 0
    p.block_q = p.block_kv = cfg.block
    p.n_init, p.window, p.step = cfg.n_init, cfg.window, cfg.step
    p.theta, p.softmax_scale = cfg.theta, cfg.softmax_scale
    p.causal, p.use_anchor = int(cfg.causal), int(cfg.use_anchor)
    p.granularity = int(cfg.granularity)
    p.engine = int(cfg.engine)
    p.dtype = {torch.float32: AA_FP32, torch.bfloat16: AA_BF16}[q.dtype]
    o = q if out is None else out
    for name, t in (("q_stride", q), ("k_stride", k), ("v_stride", v), ("o_stride", o)):
        setattr(p, name, (ctypes.c_int64 * 3)(*_strides(t, packed)))
    return p


def anchor_sizes(p: aa_params) -> aa_sizes:
    s = aa_sizes()
    _check(_lib.anchor_sizes(ctypes.byref(p), ctypes.byref(s)))
    return s


def anchor_workspace_bytes(p: aa_params) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.anchor_workspace_bytes(ctypes.byref(p), ctypes.byref(n)))
    return int(n.value)


def anchor_compute(p, q, k, v, M, L, Acc, xa_pooled, stream=None):
    _check(_lib.anchor_compute(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(M), _ptr(L), _ptr(Acc),
                               _ptr(xa_pooled), _stream(stream)))


def stripe_select(p, q, k, xa_pooled, counts, offsets, idx, overflow_flag, ws, stream=None, idx_capacity=None):
    cap = idx.numel() if idx_capacity is None else idx_capacity
    _check(_lib.stripe_select(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(xa_pooled), _ptr(counts), _ptr(offsets),
                              _ptr(idx), cap, _ptr(overflow_flag), _ptr(ws),
                              0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)))


def stripe_select_noalloc(p, q, k, xa_pooled, counts, offsets, idx, overflow_flag, stream=None, idx_capacity=None):
    """stripe_select with the library's own static scratch: no workspace argument, no allocation."""
    cap = idx.numel() if idx_capacity is None else idx_capacity
    _check(_lib.stripe_select_noalloc(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(xa_pooled), _ptr(counts),
                                      _ptr(offsets), _ptr(idx), cap, _ptr(overflow_flag), _stream(stream)))


def sparse_attn(p, q, k, v, M, L, Acc, counts, offsets, idx, out, lse=None, stream=None, idx_capacity=None):
    cap = idx.numel() if idx_capacity is None else idx_capacity
    _check(_lib.sparse_attn(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(M), _ptr(L), _ptr(Acc), _ptr(counts),
                            _ptr(offsets), _ptr(idx), cap, _ptr(out), _ptr(lse), _stream(stream)))


def anchor_attention_prefill(p, q, k, v, out, lse, stats, ws, stream=None):
    _check(_lib.anchor_attention_prefill(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
                                         _ptr(stats), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                         _stream(stream)))


def dense_causal_flash(p, q, k, v, out, lse=None, stream=None):
    _check(_lib.dense_causal_flash(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
                                   _stream(stream)))


def alloc_stage_buffers(p: aa_params, device="cuda", want_acc=True, idx_capacity=None) -> dict:
    """torch allocations sized by anchor_sizes() for the stage-wise entry points."""
    s = anchor_sizes(p)
    f32 = dict(dtype=torch.float32, device=device)
    cap = s.idx_capacity_max if idx_capacity is None else idx_capacity
    return dict(
        sizes=s,
        M=torch.empty(s.rows, **f32), L=torch.empty(s.rows, **f32),
        Acc=torch.empty(s.acc_elems, **f32) if want_acc else None,
        xa=torch.empty(s.blocks, **f32),
        counts=torch.empty(s.groups, dtype=torch.int32, device=device),
        offsets=torch.empty(s.groups + 1, dtype=torch.int64, device=device),
        idx=torch.empty(max(cap, 64), dtype=torch.int32, device=device),
        flag=torch.zeros(1, dtype=torch.int32, device=device),
        ws=torch.empty(max(s.select_ws_bytes, 256), dtype=torch.uint8, device=device),
        lse=torch.empty(s.rows, **f32),
    )


# ------------------------------------------------------------------ paged key / value cache
def alloc_kv_cache(n_pages: int, Hkv: int, page_size: int, d: int, dtype=torch.bfloat16, format=AA_KV_PLAIN, device="cuda") -> dict:
    """Pools for n_pages pages: k, v [n_pages, Hkv, page_size, d] of dtype, or for AA_KV_FP4 their codes uint8 [.., d // 2] and
    k_scale, v_scale uint8 [n_pages, Hkv, d // 32, page_size].  Cleared, though no kernel lets what is behind a sequence's end
    reach an output."""
    if format == AA_KV_PLAIN:
        k, v = (torch.zeros(n_pages, Hkv, page_size, d, dtype=dtype, device=device) for _ in range(2))
        return dict(k=k, v=v, k_scale=None, v_scale=None)
    u8 = dict(dtype=torch.uint8, device=device)
    k, v = (torch.zeros(n_pages, Hkv, page_size, d // 2, **u8) for _ in range(2))
    ks, vs = (torch.full((n_pages, Hkv, d // 32, page_size), 127, **u8) for _ in range(2))
    return dict(k=k, v=v, k_scale=ks, v_scale=vs)


_KV_FIELDS = dict(q="q_stride", k="k_stride", v="v_stride", out="o_stride", k_out="ko_stride")


def _kv_strides(t, packed):
    """Strides of a tensor of new tokens; a dimension of one entry has none that matters."""
    if t.dim() != (3 if packed else 4):
        raise ValueError("new tokens are [B, H, n, d], or [H, total, d] with cu_seqlens: got shape %s" % (tuple(t.shape),))
    if t.stride(-1) != 1:
        raise ValueError("the last dimension has to be contiguous: strides %s" % (t.stride(),))
    s = [0 if n == 1 else st for n, st in zip(t.shape[:-1], t.stride()[:-1])]
    return (ctypes.c_int64 * 3)(*(([0] if packed else []) + s))


def _pool_strides(t, unit):
    """Strides of a pool (rows of `unit` entries); for a dimension of one entry any multiple of a row."""
    s, step = [], unit
    for n, st in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        s.append(step if n == 1 else st)
        step = max(step, s[-1] * n)
    return (ctypes.c_int64 * 3)(*reversed(s))


def make_kv_params(cache: dict, page_table, kv_len, q=None, k=None, v=None, out=None, k_out=None, cu_seqlens=None, max_new=None,
                   max_len: int = 0, causal: bool = True, rot_dim: int = 0, rot_interleaved: bool = False,
                   softmax_scale: float = 0.0, Hq=None) -> aa_kv_params:
    """Describe one call on the paged cache `cache` (alloc_kv_cache, or pools of any strides with whole rows).

    page_table int32 [B, max_pages], kv_len int32 [B] (tokens of each sequence, the new ones included).  New tokens: q [B, Hq, n, d],
    k, v [B, Hkv, n, d], or with cu_seqlens (device int32 [B + 1]) packed [Hq, total, d] and [Hkv, total, d], max_new the most of any
    sequence.  kv_append: q, k, v, out (the turned queries), k_out (the turned keys).  kv_attn: q, out.  kv_read: k, v (where it
    writes).  The tensors named here are kept alive by the result; calls take tensors of the same strides."""
    named = dict(q=q, k=k, v=v, out=out, k_out=k_out)
    given = {n: t for n, t in named.items() if t is not None}
    if not given:
        raise ValueError("no tensor of new tokens: name the ones that the call takes")
    first, packed = next(iter(given.values())), cu_seqlens is not None
    p = aa_kv_params()
    p.format = AA_KV_PLAIN if cache.get("k_scale") is None else AA_KV_FP4
    p.dtype = _kv_dtype(first)
    p.n_pages, p.Hkv, p.page_size = cache["k"].shape[:3]
    p.d = first.shape[-1]
    heads = q if q is not None else out
    p.Hq = heads.shape[-3] if heads is not None else int(Hq or p.Hkv)
    p.B, p.max_pages = page_table.shape
    axis = first.shape[-2]
    p.N = int(axis if max_new is None else max_new)
    for name, t in given.items():
        want = (p.Hq if name in ("q", "out") else p.Hkv, axis, p.d)
        if tuple(t.shape) != (want if packed else (p.B,) + want) or t.dtype != first.dtype:
            raise ValueError("%s: shape %s %s, expected %s %s" % (name, tuple(t.shape), t.dtype,
                                                                want if packed else (p.B,) + want, first.dtype))
    if not packed and p.N != axis:
        raise ValueError("max_new %d of a batch with %d new tokens a sequence" % (p.N, axis))
    if p.format == AA_KV_PLAIN:
        shapes = dict(k=((p.n_pages, p.Hkv, p.page_size, p.d), first.dtype))
    else:
        shapes = dict(k=((p.n_pages, p.Hkv, p.page_size, p.d // 2), torch.uint8),
                      k_scale=((p.n_pages, p.Hkv, p.d // 32, p.page_size), torch.uint8))
    for key, (shape, dtype) in shapes.items():
        for t in (cache[key], cache[key.replace("k", "v", 1)]):
            if tuple(t.shape) != shape or t.dtype != dtype or t.stride(-1) != 1:
                raise ValueError("cache[%r]: shape %s %s, expected %s %s with contiguous rows" % (key, tuple(t.shape), t.dtype, shape, dtype))
    ints = [("page_table", page_table, (p.B, p.max_pages)), ("kv_len", kv_len, (p.B,))]
    if packed:
        ints.append(("cu_seqlens", cu_seqlens, (p.B + 1,)))
    for name, t, shape in ints:
        if t.dtype != torch.int32 or tuple(t.shape) != shape or (t.shape[-1] > 1 and t.stride(-1) != 1):
            raise ValueError("%s: shape %s %s, expected contiguous int32 %s" % (name, tuple(t.shape), t.dtype, shape))
    held = list(given.values()) + [t for t in cache.values() if t is not None] + [page_table, kv_len] + ([cu_seqlens] if packed else [])
    if any(t.device != first.device for t in held):
        raise ValueError("tensors on different devices: %s" % sorted({str(t.device) for t in held}))
    for name, t in given.items():
        setattr(p, _KV_FIELDS[name], _kv_strides(t, packed))
    p.kc, p.vc = cache["k"].data_ptr(), cache["v"].data_ptr()
    p.kc_stride, p.vc_stride = (_pool_strides(cache[x], cache[x].shape[-1]) for x in ("k", "v"))
    if p.format == AA_KV_FP4:
        p.ks, p.vs = cache["k_scale"].data_ptr(), cache["v_scale"].data_ptr()
        p.ks_stride, p.vs_stride = (_pool_strides(cache[x], p.page_size) for x in ("k_scale", "v_scale"))
    p.page_table, p.kv_len = page_table.data_ptr(), kv_len.data_ptr()
    p.table_stride = p.max_pages if p.B == 1 else page_table.stride(0)
    p.cu_seqlens = cu_seqlens.data_ptr() if packed else None
    p.total_tokens = axis if packed else 0
    p.max_len, p.causal = int(max_len), int(bool(causal))
    p.rot_dim, p.rot_interleaved, p.softmax_scale = int(rot_dim), int(bool(rot_interleaved)), softmax_scale
    p.device = first.device
    p.new_rows = axis if packed else p.B * axis
    p.made_for = {name: (t.shape, t.stride(), t.dtype, t.device) for name, t in given.items()}
    p.held = held
    return p


def _kv_dtype(t):
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("new tokens are float32 or bfloat16: got %s" % t.dtype)
    return AA_FP32 if t.dtype == torch.float32 else AA_BF16


def _kv_check(p, name, t):
    """A tensor of a call against the one that p was made for: shape, type, strides and device decide what the kernels touch."""
    if t is None:
        return None
    shape, strides, dtype, device = p.made_for.get(name, (None,) * 4)
    if t.shape != shape or t.dtype != dtype or t.device != device or (
            t.stride() != strides and tuple(_kv_strides(t, len(shape) == 3)) != tuple(getattr(p, _KV_FIELDS[name]))):
        raise ValueError("%s: %s %s strides %s on %s, but the params were made for %s %s strides %s on %s"
                         % (name, tuple(t.shape), t.dtype, t.stride(), t.device, shape and tuple(shape), dtype, strides, device))
    return t.data_ptr()


def _kv_call(fn, p, stream, *args):
    """Calls fn with p's device as the current one; a decode step is a few microseconds on the GPU, so the way there is kept short."""
    at = p.device.index
    if at is None:
        raise ValueError("the tensors are on %s: the kernels need a GPU" % p.device)
    if torch.cuda.current_device() == at:
        rc = fn(ctypes.byref(p), *args, torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(at):
            rc = fn(ctypes.byref(p), *args, torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream)
    if rc != AA_OK:
        raise AnchorError(rc)


def _at(t):
    return None if t is None else t.data_ptr()


def kv_attn_workspace_bytes(p: aa_kv_params) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.kv_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(n)))
    return int(n.value)


def kv_append(p, q, k, v, inv_freq=None, positions=None, q_out=None, k_out=None, stream=None):
    """Turn the new queries and keys by their position (q_out, k_out) and store keys and values in the cache's pages.
    inv_freq float32 [rot_dim // 2]; positions int32, one a new token ([B, n] or packed), None: its place in the sequence."""
    at = [_kv_check(p, *x) for x in (("q", q), ("k", k), ("v", v), ("out", q_out), ("k_out", k_out))]
    if p.rot_dim and (inv_freq is None or inv_freq.dtype != torch.float32 or inv_freq.numel() != p.rot_dim // 2
                      or not inv_freq.is_contiguous() or inv_freq.device != p.device):
        raise ValueError("inv_freq: contiguous float32 [%d] on %s expected" % (p.rot_dim // 2, p.device))
    if positions is not None and (positions.dtype != torch.int32 or not positions.is_contiguous() or positions.device != p.device
                                  or positions.numel() != p.new_rows):
        raise ValueError("positions: contiguous int32 on %s, one a new token (%d), expected" % (p.device, p.new_rows))
    _kv_call(_lib.kv_append, p, stream, at[0], at[1], at[2], _at(inv_freq), _at(positions), at[3], at[4])


def kv_attn(p, q, out, lse=None, ws=None, stream=None):
    """Attention of the new queries over the cached tokens that they see.  lse float32 [rows]; ws: kv_attn_workspace_bytes(p)
    bytes, of this call alone while it runs."""
    at_q, at_out = _kv_check(p, "q", q), _kv_check(p, "out", out)
    if lse is not None and (lse.dtype != torch.float32 or lse.numel() != p.Hq * p.new_rows or not lse.is_contiguous() or lse.device != p.device):
        raise ValueError("lse: contiguous float32 [%d] on %s expected" % (p.Hq * p.new_rows, p.device))
    if ws is not None and (ws.device != p.device or not ws.is_contiguous()):
        raise ValueError("ws: contiguous on %s expected" % p.device)
    _kv_call(_lib.kv_attn, p, stream, at_q, at_out, _at(lse), _at(ws), 0 if ws is None else ws.numel() * ws.element_size())


def kv_read(p, k_out=None, v_out=None, stream=None):
    """Copy the rows of every sequence's new tokens out of the cache (4 bits: their values)."""
    _kv_call(_lib.kv_read, p, stream, _kv_check(p, "k", k_out), _kv_check(p, "v", v_out))


def default_scale(d: int) -> float:
    return 1.0 / math.sqrt(d)
