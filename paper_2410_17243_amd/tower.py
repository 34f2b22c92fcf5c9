"""Operators of the text tower on AMD MI355X: Python binding of include/infcl_tower.h.

What an encoder trained beside the contrastive loss runs: token embedding,
attention over packed sequences, and activation checkpoints in 8 bits.  As in
the package itself this module only marshals arguments; the work is done by
the HIP kernels of libinfcl.so on the current stream, and nothing falls back.
The autograd functions are differentiable once: a gradient of their gradient is
an error.

Token embedding
    embed_fwd(tokens, table, scale=1.0) -> out
    embed_bwd(tokens, dout, vocab, scale=1.0, grad_dtype=None) -> dtable
    embed(tokens, table, scale=1.0) -> out   (torch.autograd.Function)
Packed attention
    packed_attn_fwd(q, k, v, cu_q, max_q, cu_k=None, max_k=None, causal=True, scale=None, need_lse=True,
                    len_k=None) -> (out, lse)
    packed_attn_bwd(q, k, v, out, lse, dout, cu_q, max_q, ...) -> (dq, dk, dv)
    packed_attn(q, k, v, cu_q, max_q, ...) -> out   (torch.autograd.Function)
    packed_attn_qkv(qkv, heads, kv_heads, cu, max_len, ...) -> out, of one projection [tokens, heads + 2 kv_heads, hd]
8-bit checkpoints (a Ckpt8 holds the bytes and the exponents)
    ckpt8_pack(x) -> Ckpt8
    ckpt8_unpack(kept) -> x^
    ckpt8_act_fwd(x, act) -> (out, Ckpt8)
    ckpt8_act_bwd(dy, kept, act) -> dx
    ckpt8_wgrad(dy, kept, act="none", grad_dtype=None) -> dw
    linear8(x, w, b=None), mlp8(x, w1, b1, w2, b2, act)   (torch.autograd.Functions)
"""

from __future__ import annotations

import ctypes
import functools

import torch
from torch.amp import custom_bwd, custom_fwd
from torch.autograd.function import once_differentiable

from . import INFCL_BF16, INFCL_F16, INFCL_F32, _check, _ptr, _raw_stream, load_library

_CODES = {torch.bfloat16: INFCL_BF16, torch.float16: INFCL_F16, torch.float32: INFCL_F32}
ACTS = {"none": 0, "gelu": 1, "quick_gelu": 2}
GROUP = 32  # features that share an exponent

_lib = None


class _Shape(ctypes.Structure):  # infcl_attn_shape
    _fields_ = [("total_q", ctypes.c_int64), ("total_k", ctypes.c_int64), ("nseq", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("max_q", ctypes.c_int64),
                ("max_k", ctypes.c_int64), ("scale", ctypes.c_float)]


class _View(ctypes.Structure):  # infcl_attn_view
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


def _load():
    """libinfcl.so with the argument types of include/infcl_tower.h set."""
    global _lib
    if _lib is None:
        lib = load_library()
        i64, sz, vp, ip, fl = ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int, ctypes.c_float
        psz = ctypes.POINTER(sz)
        for name, args in {
            "infcl_embed_fwd": [vp, ip, i64, vp, i64, i64, ip, fl, vp, vp],
            "infcl_embed_bwd_workspace": [i64, i64, i64, psz],
            "infcl_embed_bwd": [vp, ip, i64, vp, i64, i64, ip, fl, vp, ip, vp, sz, vp],
            "infcl_attn_workspace": [ctypes.POINTER(_Shape), psz, psz],
            "infcl_attn_fwd": [ctypes.POINTER(_Shape), _View, _View, _View, vp, vp, vp, _View, vp, vp, sz, vp],
            "infcl_attn_bwd": [ctypes.POINTER(_Shape), _View, _View, _View, vp, vp, _View, vp, _View, _View, _View,
                               _View, vp, sz, vp],
            "infcl_ckpt8_pack": [vp, i64, i64, i64, ip, vp, vp, vp],
            "infcl_ckpt8_unpack": [vp, vp, i64, i64, ip, vp, vp],
            "infcl_ckpt8_act_fwd": [vp, i64, i64, i64, ip, ip, vp, vp, vp, vp],
            "infcl_ckpt8_act_bwd": [vp, i64, vp, vp, i64, i64, ip, ip, vp, vp],
            "infcl_ckpt8_wgrad_workspace": [i64, i64, i64, psz],
            "infcl_ckpt8_wgrad": [vp, i64, vp, vp, i64, i64, i64, ip, ip, vp, ip, vp, sz, vp],
        }.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, ip
        _lib = lib
    return _lib


def _device(*named):
    """The one device of the given (name, tensor) pairs."""
    dev = named[0][1].device
    for name, t in named:
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        if t.device != dev:
            raise ValueError(f"{named[0][0]} and {name} must be on one device, got {dev} and {t.device}")
    return dev


def _code(t, name):
    c = _CODES.get(t.dtype)
    if c is None:
        raise TypeError(f"{name} must be bfloat16, float16 or float32, got {t.dtype}")
    return c


# Small calls are bound by host time (an activation of 9 x 64: 12 us of it, 4 of
# them the library's), so what depends on sizes alone is asked for once for each
# set of them.

@functools.lru_cache(maxsize=4096)
def _workspace_bytes(name, *sizes) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(_load(), name)(*sizes, ctypes.byref(n)), name)
    return max(n.value, 256)


def _workspace(name, dev, *sizes):
    return torch.empty(_workspace_bytes(name, *sizes), dtype=torch.uint8, device=dev)


# ------------------------------------------------------------ token embedding

def _tokens(tokens):
    if tokens.dtype == torch.int32:
        size = 4
    elif tokens.dtype == torch.int64:
        size = 8
    else:
        raise TypeError(f"tokens must be int32 or int64, got {tokens.dtype}")
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")
    return size


def embed_fwd(tokens, table, scale: float = 1.0):
    """scale * table[tokens], [*tokens.shape, d]; rows of tokens outside the table are zero."""
    dev = _device(("tokens", tokens), ("table", table))
    size, code = _tokens(tokens), _code(table, "table")
    if table.dim() != 2 or not table.is_contiguous():
        raise ValueError(f"table must be contiguous [vocab, d], got {tuple(table.shape)}")
    vocab, d = table.shape
    out = torch.empty((*tokens.shape, d), dtype=table.dtype, device=dev)
    _check(_load().infcl_embed_fwd(tokens.data_ptr(), size, tokens.numel(), table.data_ptr(), vocab, d, code,
                                   float(scale), out.data_ptr(), _raw_stream(dev)), "infcl_embed_fwd")
    return out


def embed_bwd(tokens, dout, vocab: int, scale: float = 1.0, grad_dtype=None):
    """The table's gradient [vocab, d] (every row written), of grad_dtype:
    float32 (default) or dout's dtype."""
    dev = _device(("tokens", tokens), ("dout", dout))
    size, code = _tokens(tokens), _code(dout, "dout")
    if dout.shape[:-1] != tokens.shape or not dout.is_contiguous():
        raise ValueError(f"dout must be contiguous [*tokens.shape, d], got {tuple(dout.shape)} for {tuple(tokens.shape)}")
    gdt = torch.float32 if grad_dtype is None else grad_dtype
    if gdt not in (torch.float32, dout.dtype):
        raise TypeError(f"grad_dtype must be float32 or dout's dtype {dout.dtype}, got {gdt}")
    n, d = tokens.numel(), dout.shape[-1]
    lib = _load()
    ws = _workspace("infcl_embed_bwd_workspace", dev, n, int(vocab), d)
    dtable = torch.empty((int(vocab), d), dtype=gdt, device=dev)
    _check(lib.infcl_embed_bwd(tokens.data_ptr(), size, n, dout.data_ptr(), int(vocab), d, code, float(scale),
                               dtable.data_ptr(), _CODES[gdt], ws.data_ptr(), ws.numel(), _raw_stream(dev)),
           "infcl_embed_bwd")
    return dtable


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, table, scale):
        ctx.save_for_backward(tokens)
        ctx.vocab, ctx.scale = table.shape[0], scale
        return embed_fwd(tokens, table, scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        (tokens,) = ctx.saved_tensors
        return None, embed_bwd(tokens, dout.contiguous(), ctx.vocab, ctx.scale, dout.dtype), None


def embed(tokens, table, scale: float = 1.0):
    """scale * table[tokens]; differentiable with respect to the table (up to 2^26
    tokens)."""
    if table.requires_grad and torch.is_grad_enabled() and table.dim() == 2:  # (the gradient's limits, before the work)
        _workspace_bytes("infcl_embed_bwd_workspace", tokens.numel(), *table.shape)
    return _Embed.apply(tokens, table, float(scale))


# ----------------------------------------------------------- packed attention

@functools.lru_cache(maxsize=4096)
def _plan(*fields):
    """(infcl_attn_shape, workspace bytes of the forward and of the backward) for its fields."""
    sh, f, b = _Shape(*fields), ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(_load().infcl_attn_workspace(ctypes.byref(sh), ctypes.byref(f), ctypes.byref(b)), "infcl_attn_workspace")
    return ctypes.byref(sh), f.value, b.value


def _heads_view(t, name, like=None):
    """t as [tokens, heads, head_dim] with features next to each other and rows of
    16-byte units (strides of dimensions of one or no entry do not matter)."""
    shape, strides = t.shape, t.stride()
    if len(shape) != 3 or strides[2] != 1 and shape[2] > 1:
        raise ValueError(f"{name} must be [tokens, heads, head_dim] with contiguous features, got {tuple(shape)}, "
                         f"strides {strides}")
    if like is not None and t.dtype != like.dtype:
        raise ValueError(f"{name} must be {like.dtype}, got {t.dtype}")
    return _View(t.data_ptr(), strides[0] if shape[0] > 1 else shape[1] * shape[2], strides[1] if shape[1] > 1 else 0)


def _cu(cu, name, dev):
    if cu.dtype != torch.int32 or cu.dim() != 1 or cu.numel() < 1 or not cu.is_contiguous() or cu.device != dev:
        raise ValueError(f"{name} must be a contiguous int32 vector on {dev}, got {cu.dtype} "
                         f"{tuple(cu.shape)} on {cu.device}")


def _attn_call(q, k, v, cu_q, max_q, cu_k, max_k, causal, scale):
    """Checks the arguments; (device, plan, views of q, k and v, cu_k)."""
    dev = _device(("q", q), ("k", k), ("v", v))
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError(f"q must be bfloat16 or float16, got {q.dtype}")
    vq, vk, vv = _heads_view(q, "q"), _heads_view(k, "k", q), _heads_view(v, "v", q)
    tq, heads, hd = q.shape
    tk, kv, khd = k.shape
    if k.shape != v.shape or khd != hd or kv < 1 or heads % kv:
        raise ValueError(f"k and v must be [tokens, kv_heads, {hd}], kv_heads a divisor of {heads}, got "
                         f"{tuple(k.shape)}, {tuple(v.shape)}")
    _cu(cu_q, "cu_q", dev)
    if cu_k is None:
        if tk != tq:
            raise ValueError(f"without cu_k there are as many keys as queries, got {tk} and {tq}")
        cu_k, max_k = cu_q, max_q
    else:
        _cu(cu_k, "cu_k", dev)
        if cu_k.numel() != cu_q.numel():
            raise ValueError(f"cu_q and cu_k must have as many entries, got {cu_q.numel()} and {cu_k.numel()}")
        if max_k is None:
            raise ValueError("cu_k comes with max_k")
    plan = _plan(tq, tk, cu_q.numel() - 1, heads, kv, hd, _CODES[q.dtype], 1 if causal else 0, int(max_q), int(max_k),
                 hd ** -0.5 if scale is None else float(scale))
    return dev, plan, vq, vk, vv, cu_k


def packed_attn_fwd(q, k, v, cu_q, max_q: int, cu_k=None, max_k=None, causal: bool = True, scale=None,
                    need_lse: bool = True, len_k=None):
    """Attention over packed sequences: q [tokens, heads, head_dim], k, v [tokens,
    kv_heads, head_dim]; sequence z has the rows cu_q[z] .. cu_q[z+1] of q and
    cu_k[z] .. cu_k[z+1] (cu_q's without cu_k) of k and v.  max_q, max_k: the longest
    lengths.  Returns out [tokens, heads, head_dim] and lse [heads, tokens] float32
    (None without need_lse).  scale: 1 / sqrt(head_dim) by default.  len_k [sequences]
    int32: the keys in use, where cu_k gives each sequence room for more."""
    dev, (sh, n, _), vq, vk, vv, cu_k = _attn_call(q, k, v, cu_q, max_q, cu_k, max_k, causal, scale)
    if len_k is not None:
        _cu(len_k, "len_k", dev)
        if len_k.numel() != cu_q.numel() - 1:
            raise ValueError(f"len_k must have an entry for each of {cu_q.numel() - 1} sequences, got {len_k.numel()}")
    tq, heads, hd = q.shape
    out = torch.empty((tq, heads, hd), dtype=q.dtype, device=dev)
    lse = torch.empty((heads, tq), dtype=torch.float32, device=dev) if need_lse else None
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _check(_load().infcl_attn_fwd(sh, vq, vk, vv, cu_q.data_ptr(), cu_k.data_ptr(), _ptr(len_k),
                                  _View(out.data_ptr(), heads * hd, hd), _ptr(lse), _ptr(ws), n, _raw_stream(dev)),
           "infcl_attn_fwd")
    return out, lse


def packed_attn_bwd(q, k, v, out, lse, dout, cu_q, max_q: int, cu_k=None, max_k=None, causal: bool = True, scale=None,
                    grads=None):
    """dq, dk, dv of packed_attn_fwd without len_k (every key between cu_k's offsets counts
    as in use); written into grads = (dq, dk, dv) where given."""
    dev, (sh, _, n), vq, vk, vv, cu_k = _attn_call(q, k, v, cu_q, max_q, cu_k, max_k, causal, scale)
    _device(("q", q), ("out", out), ("lse", lse), ("dout", dout))
    if out.shape != q.shape or dout.shape != q.shape:
        raise ValueError(f"out and dout must be {tuple(q.shape)}, got {tuple(out.shape)}, {tuple(dout.shape)}")
    if lse.shape != (q.shape[1], q.shape[0]) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError(f"lse must be contiguous float32 [heads, tokens], got {lse.dtype} {tuple(lse.shape)}")
    if grads is None:
        dq, dk, dv = (torch.empty(t.shape, dtype=q.dtype, device=dev) for t in (q, k, v))
    else:
        dq, dk, dv = grads
        _device(("q", q), ("dq", dq), ("dk", dk), ("dv", dv))
        if dq.shape != q.shape or dk.shape != k.shape or dv.shape != v.shape:
            raise ValueError("grads must have the shapes of q, k and v")
    ws = torch.empty(n, dtype=torch.uint8, device=dev)
    _check(_load().infcl_attn_bwd(sh, vq, vk, vv, cu_q.data_ptr(), cu_k.data_ptr(), _heads_view(out, "out", q),
                                  lse.data_ptr(), _heads_view(dout, "dout", q), _heads_view(dq, "dq", q),
                                  _heads_view(dk, "dk", q), _heads_view(dv, "dv", q), ws.data_ptr(), n,
                                  _raw_stream(dev)), "infcl_attn_bwd")
    return dq, dk, dv


class _PackedAttn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_q, max_q, cu_k, max_k, causal, scale):
        out, lse = packed_attn_fwd(q, k, v, cu_q, max_q, cu_k, max_k, causal, scale)
        ctx.save_for_backward(q, k, v, out, lse, cu_q, cu_k)
        ctx.rest = (max_q, max_k, causal, scale)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, cu_q, cu_k = ctx.saved_tensors
        max_q, max_k, causal, scale = ctx.rest
        return (*packed_attn_bwd(q, k, v, out, lse, dout.contiguous(), cu_q, max_q, cu_k, max_k, causal, scale),
                None, None, None, None, None, None)


def packed_attn(q, k, v, cu_q, max_q: int, cu_k=None, max_k=None, causal: bool = True, scale=None):
    """packed_attn_fwd's out; differentiable with respect to q, k and v."""
    return _PackedAttn.apply(q, k, v, cu_q, max_q, cu_k, max_k, causal, scale)


class _PackedAttnQkv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, heads, kv_heads, cu, max_len, causal, scale):
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        out, lse = packed_attn_fwd(q, k, v, cu, max_len, causal=causal, scale=scale)
        ctx.save_for_backward(qkv, out, lse, cu)
        ctx.rest = (heads, kv_heads, max_len, causal, scale)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        qkv, out, lse, cu = ctx.saved_tensors
        heads, kv_heads, max_len, causal, scale = ctx.rest
        a, b = heads, heads + kv_heads
        d = torch.empty(qkv.shape, dtype=qkv.dtype, device=qkv.device)
        packed_attn_bwd(qkv[:, :a], qkv[:, a:b], qkv[:, b:], out, lse, dout.contiguous(), cu, max_len, causal=causal,
                        scale=scale, grads=(d[:, :a], d[:, a:b], d[:, b:]))
        return d, None, None, None, None, None, None


def packed_attn_qkv(qkv, heads: int, kv_heads: int, cu, max_len: int, causal: bool = True, scale=None):
    """packed_attn of one projection's output qkv [tokens, heads + 2 kv_heads,
    head_dim] (q, then k, then v), whose gradient comes as one array too."""
    if qkv.dim() != 3 or qkv.shape[1] != heads + 2 * kv_heads:
        raise ValueError(f"qkv must be [tokens, {heads} + 2 * {kv_heads}, head_dim], got {tuple(qkv.shape)}")
    return _PackedAttnQkv.apply(qkv, heads, kv_heads, cu, max_len, causal, scale)


# --------------------------------------------------------- 8-bit checkpoints

class Ckpt8:
    """An activation [*, d] kept in 8 bits: q (int8, its shape), exps (uint8, a
    byte for every 32 features of a row), and the dtype it had."""

    __slots__ = ("q", "exps", "dtype")

    def __init__(self, q, exps, dtype):
        self.q, self.exps, self.dtype = q, exps, dtype

    @property
    def shape(self):
        return self.q.shape

    def nbytes(self):
        return self.q.numel() + self.exps.numel()


def _rows(t, name):
    """(rows, features, row stride) of a tensor whose leading dimensions are one
    sequence of evenly spaced rows."""
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError(f"{name} must be [*, d], got {tuple(t.shape)}")
    d = t.shape[-1]
    if t.is_contiguous():
        return t.numel() // d, d, d
    if t.dim() != 2 or t.stride(1) != 1 or t.stride(0) < d:
        raise ValueError(f"{name} must be contiguous, or rows [n, d] of a wider array")
    return t.shape[0], d, t.stride(0)


def _act(act, allow_none=False):
    a = ACTS.get(act)
    if a is None or (a == 0 and not allow_none):
        raise ValueError(f"act must be one of {[k for k in ACTS if allow_none or k != 'none']}, got {act!r}")
    return a


def _kept_for(x, d, dev):
    q = torch.empty(x.shape, dtype=torch.int8, device=dev)
    return Ckpt8(q, torch.empty((*x.shape[:-1], (d + GROUP - 1) // GROUP), dtype=torch.uint8, device=dev), x.dtype)


def _check_kept(kept):
    q, e = kept.q, kept.exps
    if q.dtype != torch.int8 or e.dtype != torch.uint8 or not q.is_contiguous() or not e.is_contiguous():
        raise ValueError("a checkpoint holds contiguous int8 values and uint8 exponents")
    if e.shape != (*q.shape[:-1], (q.shape[-1] + GROUP - 1) // GROUP):
        raise ValueError(f"exponents {tuple(e.shape)} do not fit values {tuple(q.shape)}")


def ckpt8_pack(x) -> Ckpt8:
    """x [*, d] in 8 bits with a power of two for every 32 features."""
    dev, code = _device(("x", x)), _code(x, "x")
    n, d, stride = _rows(x, "x")
    kept = _kept_for(x, d, dev)
    _check(_load().infcl_ckpt8_pack(x.data_ptr(), stride, n, d, code, kept.q.data_ptr(), kept.exps.data_ptr(),
                                    _raw_stream(dev)), "infcl_ckpt8_pack")
    return kept


def ckpt8_unpack(kept: Ckpt8):
    """What the checkpoint stands for, in the dtype x had."""
    _check_kept(kept)
    dev = _device(("values", kept.q), ("exponents", kept.exps))
    out = torch.empty(kept.q.shape, dtype=kept.dtype, device=dev)
    n, d, _ = _rows(kept.q, "values")
    _check(_load().infcl_ckpt8_unpack(kept.q.data_ptr(), kept.exps.data_ptr(), n, d, _CODES[kept.dtype],
                                      out.data_ptr(), _raw_stream(dev)), "infcl_ckpt8_unpack")
    return out


def ckpt8_act_fwd(x, act: str):
    """(f(x), the checkpoint of x) in one pass; act: "gelu" or "quick_gelu"."""
    dev, code, a = _device(("x", x)), _code(x, "x"), _act(act)
    n, d, stride = _rows(x, "x")
    kept = _kept_for(x, d, dev)
    out = torch.empty(x.shape, dtype=x.dtype, device=dev)
    _check(_load().infcl_ckpt8_act_fwd(x.data_ptr(), stride, n, d, code, a, out.data_ptr(), kept.q.data_ptr(),
                                       kept.exps.data_ptr(), _raw_stream(dev)), "infcl_ckpt8_act_fwd")
    return out, kept


def ckpt8_act_bwd(dy, kept: Ckpt8, act: str):
    """dy f'(x^)."""
    _check_kept(kept)
    dev, a = _device(("dy", dy), ("values", kept.q), ("exponents", kept.exps)), _act(act)
    if dy.shape != kept.q.shape or dy.dtype != kept.dtype:
        raise ValueError(f"dy must be {tuple(kept.q.shape)} of {kept.dtype}, got {tuple(dy.shape)} of {dy.dtype}")
    n, d, stride = _rows(dy, "dy")
    dx = torch.empty(dy.shape, dtype=dy.dtype, device=dev)
    _check(_load().infcl_ckpt8_act_bwd(dy.data_ptr(), stride, kept.q.data_ptr(), kept.exps.data_ptr(), n, d,
                                       _CODES[kept.dtype], a, dx.data_ptr(), _raw_stream(dev)), "infcl_ckpt8_act_bwd")
    return dx


def ckpt8_wgrad(dy, kept: Ckpt8, act: str = "none", grad_dtype=None):
    """dw [m, d] = dy^T f(x^) for dy [*, m]: the weight gradient of y = f(x) w^T.
    dy is bfloat16 or float16; grad_dtype is float32 (default) or dy's dtype."""
    _check_kept(kept)
    dev, a = _device(("dy", dy), ("values", kept.q), ("exponents", kept.exps)), _act(act, True)
    if dy.shape[:-1] != kept.q.shape[:-1]:
        raise ValueError(f"dy {tuple(dy.shape)} and the checkpoint {tuple(kept.q.shape)} must have the same rows")
    if dy.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError(f"dy must be bfloat16 or float16, got {dy.dtype}")
    gdt = torch.float32 if grad_dtype is None else grad_dtype
    if gdt not in (torch.float32, dy.dtype):
        raise TypeError(f"grad_dtype must be float32 or dy's dtype {dy.dtype}, got {gdt}")
    n, m, stride = _rows(dy, "dy")
    d = kept.q.shape[-1]
    lib = _load()
    ws = _workspace("infcl_ckpt8_wgrad_workspace", dev, n, d, m)
    dw = torch.empty((m, d), dtype=gdt, device=dev)
    _check(lib.infcl_ckpt8_wgrad(dy.data_ptr(), stride, kept.q.data_ptr(), kept.exps.data_ptr(), n, d, m,
                                 _CODES[dy.dtype], a, dw.data_ptr(), _CODES[gdt], ws.data_ptr(), ws.numel(),
                                 _raw_stream(dev)), "infcl_ckpt8_wgrad")
    return dw


def _check_learning(name, x, *weights):
    """What the weight gradients will ask for, asked before the forward's work."""
    if not torch.is_grad_enabled():
        return
    dtype = torch.get_autocast_dtype("cuda") if torch.is_autocast_enabled("cuda") else x.dtype
    for w in weights:
        if not w.requires_grad:
            continue
        if dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"{name}: a layer learns from products in bfloat16 or float16, got {dtype}")
        if w.shape[0] % 8:
            raise ValueError(f"{name}: a layer that learns has a multiple of 8 outputs, got {w.shape[0]}")


class _Linear8(torch.autograd.Function):
    @staticmethod
    @custom_fwd(device_type="cuda")
    def forward(ctx, x, w, b):
        kept = ckpt8_pack(x)
        ctx.save_for_backward(kept.q, kept.exps, w)
        ctx.has_b = b is not None
        return torch.nn.functional.linear(x, w, b)

    @staticmethod
    @once_differentiable
    @custom_bwd(device_type="cuda")  # (the plain products as the forward's, under autocast too)
    def backward(ctx, dy):
        q, exps, w = ctx.saved_tensors
        dy = dy.contiguous()
        dx = torch.matmul(dy, w) if ctx.needs_input_grad[0] else None
        dw = ckpt8_wgrad(dy, Ckpt8(q, exps, dy.dtype), grad_dtype=dy.dtype) if ctx.needs_input_grad[1] else None
        db = dy.reshape(-1, dy.shape[-1]).sum(0) if ctx.has_b and ctx.needs_input_grad[2] else None
        return dx, dw, db


def linear8(x, w, b=None):
    """x w^T + b with x kept for the backward pass in 8 bits.  x, w (and b) of one
    16-bit dtype, or of any under autocast; the plain products are torch's, the
    weight gradient is ckpt8_wgrad's (a multiple of 8 outputs)."""
    _check_learning("linear8", x, w)
    return _Linear8.apply(x, w, b)


class _Mlp8(torch.autograd.Function):
    @staticmethod
    @custom_fwd(device_type="cuda")
    def forward(ctx, x, w1, b1, w2, b2, act):
        kx = ckpt8_pack(x)
        a, kh = ckpt8_act_fwd(torch.nn.functional.linear(x, w1, b1), act)
        ctx.save_for_backward(kx.q, kx.exps, kh.q, kh.exps, w1, w2)
        ctx.act, ctx.has_b1, ctx.has_b2 = act, b1 is not None, b2 is not None
        return torch.nn.functional.linear(a, w2, b2)

    @staticmethod
    @once_differentiable
    @custom_bwd(device_type="cuda")  # (the plain products as the forward's, under autocast too)
    def backward(ctx, dy):
        xq, xe, hq, he, w1, w2 = ctx.saved_tensors
        dy = dy.contiguous()
        kh = Ckpt8(hq, he, dy.dtype)
        dw2 = ckpt8_wgrad(dy, kh, ctx.act, dy.dtype) if ctx.needs_input_grad[3] else None
        db2 = dy.reshape(-1, dy.shape[-1]).sum(0) if ctx.has_b2 and ctx.needs_input_grad[4] else None
        dh = ckpt8_act_bwd(torch.matmul(dy, w2), kh, ctx.act)
        dw1 = ckpt8_wgrad(dh, Ckpt8(xq, xe, dy.dtype), grad_dtype=dy.dtype) if ctx.needs_input_grad[1] else None
        db1 = dh.reshape(-1, dh.shape[-1]).sum(0) if ctx.has_b1 and ctx.needs_input_grad[2] else None
        dx = torch.matmul(dh, w1) if ctx.needs_input_grad[0] else None
        return dx, dw1, db1, dw2, db2, None


def mlp8(x, w1, b1, w2, b2, act: str = "gelu"):
    """f(x w1^T + b1) w2^T + b2, which keeps x and the first product in 8 bits for
    the backward pass and nothing else (f of it is taken again from there).  Types
    and widths as for linear8."""
    _act(act)
    _check_learning("mlp8", x, w1, w2)
    return _Mlp8.apply(x, w1, b1, w2, b2, act)
