"""Operators around an encoder block's attention on AMD MI355X: Python binding of
include/infcl_block.h.

What the blocks of an encoder trained beside the contrastive loss run besides the
operators of tower.py: rotary positions, dropout, residual sums with their norms, and
layers on 8-bit floats.  As there, this module only marshals arguments; the work is
done by the HIP kernels of libinfcl.so on the current stream, and nothing falls back.
The autograd functions are differentiable once: a gradient of their gradient is an
error, and so is a forward-mode derivative.  torch.jit.trace records their calls, with
the options and whether gradients were on.  They may be captured into a HIP graph with
their backward pass, while no eager graph of the same leaves is alive (as torch asks of
every captured backward pass).

Rotary positions
    rotary_freqs(sections, base=10000.0) -> freqs
    rotary_fwd(x, pos, freqs, sections=None, turned=None, paired="halves") -> out
    rotary_bwd(dout, ...) -> dx
    rotary(x, ...) -> out   (torch.autograd.Function)
Dropout
    dropout_fwd(x, p, seed, site=0, row0=0) -> out
    dropout_bwd(dy, p, seed, ...) -> dx
    dropout(x, p, seed, ...) -> out   (torch.autograd.Function)
Residual norms
    add_norm_fwd(x, y=None, gate=, post_w=, post_b=, pre_w=, pre_b=, norm=, eps=, alpha=, p=, seed=, site=, row0=)
        -> (h, z, kept)
    add_norm_bwd(dh, dz, kept) -> (dx, dy, dgate, dpost_w, dpost_b, dpre_w, dpre_b)
    add_norm(x, y=None, ...) -> (h, z)   (torch.autograd.Function)
8-bit floats (an Fp8 holds the bytes and the exponents of 128 entries each)
    fp8_pack(x) -> Fp8, fp8_pack_both(x) -> (Fp8 of x, Fp8 of its transpose)
    fp8_unpack(packed) -> x^
    fp8_matmul(a, b, bias=None, dtype=None) -> a b^T + bias
    linear_fp8_fwd(x, w, b=None) -> (y, kept), linear_fp8_bwd(dy, kept) -> (dx, dw, db)
    linear_fp8(x, w, b=None) -> y, w a tensor (torch.autograd.Function) or an Fp8
"""

from __future__ import annotations

import ctypes
import functools

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import _check, _ptr, _raw_stream, load_library
from .tower import _CODES, _View, _code, _device, _heads_view, _rows

PAIRED = {"halves": 0, "neighbours": 1}
NORMS = {"layer": 0, "rms": 1}
BLOCK = 128  # entries that share an exponent

_lib = None
_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class _Rotary(ctypes.Structure):  # infcl_rotary_shape
    _fields_ = [("n", _i64), ("heads", _i32), ("turned", _i32), ("head_dim", _i32), ("dtype", _i32), ("paired", _i32),
                ("back", _i32), ("axes", _i32), ("pos_dtype", _i32), ("sections", _i32 * 4), ("pos_stride", _i64)]


class _Drop(ctypes.Structure):  # infcl_drop
    _fields_ = [("seed_ptr", _vp), ("seed", ctypes.c_uint64), ("row0", _i64), ("site", ctypes.c_uint32), ("p", _f32)]


class _AddNorm(ctypes.Structure):  # infcl_add_norm
    _fields_ = [("n", _i64), ("d", _i64), ("dtype", _i32), ("wdtype", _i32), ("norm", _i32), ("eps", _f32),
                ("alpha", _f32), ("drop", _Drop), ("x_stride", _i64), ("y_stride", _i64), ("gate", _vp),
                ("post_w", _vp), ("post_b", _vp), ("pre_w", _vp), ("pre_b", _vp)]


class _AddNormGrads(ctypes.Structure):  # infcl_add_norm_grads
    _fields_ = [("dh", _vp), ("dz", _vp), ("dh_stride", _i64), ("dz_stride", _i64), ("dx", _vp), ("dy", _vp),
                ("dgate", _vp), ("dpost_w", _vp), ("dpost_b", _vp), ("dpre_w", _vp), ("dpre_b", _vp)]


def _load():
    """libinfcl.so with the argument types of include/infcl_block.h set."""
    global _lib
    if _lib is None:
        lib = load_library()
        i64, sz, vp, ip = _i64, ctypes.c_size_t, _vp, ctypes.c_int
        psz, pn = ctypes.POINTER(sz), ctypes.POINTER(_AddNorm)
        for name, args in {
            "infcl_rotary": [ctypes.POINTER(_Rotary), _View, _View, vp, vp, vp],
            "infcl_dropout": [vp, i64, i64, i64, ip, _Drop, vp, vp],
            "infcl_add_norm_fwd": [pn, vp, vp, vp, vp, vp, vp],
            "infcl_add_norm_bwd_workspace": [pn, psz],
            "infcl_add_norm_bwd": [pn, vp, vp, vp, ctypes.POINTER(_AddNormGrads), vp, sz, vp],
            "infcl_fp8_pack_workspace": [i64, i64, psz],
            "infcl_fp8_pack": [vp, i64, i64, i64, ip, vp, vp, vp, vp, vp, vp, sz, vp],
            "infcl_fp8_unpack": [vp, vp, i64, i64, ip, vp, vp],
            "infcl_fp8_matmul_workspace": [i64, i64, i64, psz],
            "infcl_fp8_matmul": [vp, vp, i64, vp, vp, i64, i64, vp, ip, vp, vp, sz, vp],
            "infcl_fp8_linear_workspace": [i64, i64, i64, psz],
            "infcl_fp8_layer_sizes": [i64, i64, i64, ip, psz, psz, psz],
            "infcl_fp8_layer_fwd": [vp, i64, i64, i64, vp, i64, i64, vp, ip, ip, vp, vp, vp, sz, vp],
            "infcl_fp8_layer_bwd": [vp, i64, i64, i64, i64, ip, ip, vp, vp, vp, vp, vp, sz, vp],
            "infcl_fp8_linear": [vp, i64, i64, i64, vp, vp, i64, vp, ip, vp, vp, sz, vp],
        }.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, ip
        _lib = lib
    return _lib


def _call(name, dev, *args):
    """The entry point on dev's current stream, launched with dev as the current device."""
    fn = getattr(_load(), name)
    if torch._C._cuda_getDevice() == dev.index:
        status = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _raw_stream(dev))
    _check(status, name)


@functools.lru_cache(maxsize=4096)
def _bytes(name, *sizes) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(_load(), name)(*sizes, ctypes.byref(n)), name)
    return n.value


def _where(names, tensors):
    """The one device of the tensors that are there, the first of which is (small calls are
    bound by host time: _device names what is wrong)."""
    dev = tensors[0].device
    if dev.type == "cuda":
        for t in tensors:
            if t is not None and t.device != dev:
                break
        else:
            return dev
    return _device(*((k, t) for k, t in zip(names, tensors) if t is not None))


def _like(x):
    """Room for x's entries, rows next to each other (a microsecond less than naming its
    shape, type and device)."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


def _scratch(n, dev):
    return torch.empty(n, dtype=torch.uint8, device=dev) if n else None


# ------------------------------------------------------------ rotary positions

def rotary_freqs(sections, base: float = 10000.0, device="cuda"):
    """base^(-i / s) for i < s of each section s: the frequencies of its axis's pairs."""
    sections = (sections,) if isinstance(sections, int) else tuple(sections)
    return torch.cat([base ** (-torch.arange(s, dtype=torch.float64) / s) for s in sections]).float().to(device)


@functools.lru_cache(maxsize=4096)
def _rotary_plan(n, heads, hd, code, turned, paired, back, axes, pos_f32, stride, pairs, sections):
    """infcl_rotary_shape for these sizes."""
    if sections is None:
        sections = (pairs,)
    sections = (sections,) if isinstance(sections, int) else tuple(int(s) for s in sections)
    if len(sections) != axes or not 1 <= axes <= 4 or sum(sections) != pairs:
        raise ValueError(f"sections must be the pairs of each of {axes} axes (1 to 4), {pairs} in all, got {sections}")
    if paired not in PAIRED:
        raise ValueError(f"paired must be one of {list(PAIRED)}, got {paired!r}")
    turned = heads if turned is None else int(turned)
    if not 0 <= turned <= heads:
        raise ValueError(f"turned must be 0 to {heads} heads, got {turned}")
    return ctypes.byref(_Rotary(n, heads, turned, hd, code, PAIRED[paired], back, axes, pos_f32, (_i32 * 4)(*sections), stride))


def _turn(x, pos, freqs, sections, turned, paired, back, name):
    dev = _where((name, "pos", "freqs"), (x, pos, freqs))
    code, view = _code(x, name), _heads_view(x, name)
    n, heads, hd = x.shape
    if pos.dtype not in (torch.int32, torch.float32):
        raise TypeError(f"pos must be int32 or float32, got {pos.dtype}")
    shape, stride = pos.shape, pos.stride()
    if len(shape) not in (1, 2) or shape[0] != n or len(shape) == 2 and stride[1] != 1 and shape[1] > 1:
        raise ValueError(f"pos must be [{n}] or [{n}, axes] with a token's positions next to each other, got "
                         f"{tuple(shape)}, strides {stride}")
    if freqs.dtype != torch.float32 or freqs.dim() != 1 or not freqs.is_contiguous():
        raise ValueError(f"freqs must be a contiguous float32 vector, got {freqs.dtype} {tuple(freqs.shape)}")
    plan = _rotary_plan(n, heads, hd, code, turned, paired, back, 1 if len(shape) == 1 else shape[1],
                        int(pos.dtype == torch.float32), stride[0] if n > 1 else 0, freqs.shape[0],
                        tuple(sections) if isinstance(sections, list) else sections)
    out = _like(x)
    if n:
        _call("infcl_rotary", dev, plan, view, _View(out.data_ptr(), heads * hd, hd), pos.data_ptr(), freqs.data_ptr())
    return out


def rotary_fwd(x, pos, freqs, sections=None, turned=None, paired: str = "halves"):
    """x [tokens, heads, head_dim] (a view with contiguous features) with pairs of its
    features turned by position times frequency.  pos [tokens] or [tokens, axes], int32
    or float32; freqs [pairs] float32; sections: the pairs of each axis, in order (all of
    one axis by default).  A pair is features (f, f + pairs), "halves", or (2f, 2f + 1),
    "neighbours"; features past them and heads from `turned` on are copied."""
    return _turn(x, pos, freqs, sections, turned, paired, 0, "x")


def rotary_bwd(dout, pos, freqs, sections=None, turned=None, paired: str = "halves"):
    """The gradient of rotary_fwd: turned back."""
    return _turn(dout, pos, freqs, sections, turned, paired, 1, "dout")


class _RotaryFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, freqs, sections, turned, paired):
        ctx.save_for_backward(pos, freqs)
        ctx.rest = (sections, turned, paired)
        return rotary_fwd(x, pos, freqs, sections, turned, paired)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        return (rotary_bwd(dout.contiguous(), *ctx.saved_tensors, *ctx.rest), None, None, None, None, None)


def rotary(x, pos, freqs, sections=None, turned=None, paired: str = "halves"):
    """rotary_fwd's out; differentiable with respect to x (positions and frequencies are
    constants).  The queries and keys of a projection at once: rotary(qkv, ...,
    turned=heads + kv_heads), then packed_attn_qkv."""
    return _RotaryFn.apply(x, pos, freqs, sections, turned, paired)


# --------------------------------------------------------------------- dropout

def _drop(p, seed, site, row0, dev):
    p, site, row0 = float(p), int(site), int(row0)
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"p must be from 0 to 1, got {p}")
    if not 0 <= site < 1 << 32 or not 0 <= row0 < 1 << 62:
        raise ValueError(f"site must be below 2^32 and row0 below 2^62, both from 0 on, got {site} and {row0}")
    if isinstance(seed, torch.Tensor):
        if seed.dtype != torch.int64 or seed.numel() != 1 or seed.device != dev:
            raise ValueError(f"seed must be an int or an int64 tensor of one element on {dev}, got {seed.dtype} "
                             f"{tuple(seed.shape)} on {seed.device}")
        return _Drop(seed.data_ptr(), 0, row0, site, p)
    return _Drop(None, int(seed) & (1 << 64) - 1, row0, site, p)


def _dropped(x, p, seed, site, row0, name):
    dev, code = _where((name,), (x,)), _code(x, name)
    n, d, stride = _rows(x, name)
    drop = _drop(p, seed, site, row0, dev)
    out = _like(x)
    _call("infcl_dropout", dev, x.data_ptr(), stride, n, d, code, drop, out.data_ptr())
    return out


def dropout_fwd(x, p: float, seed, site: int = 0, row0: int = 0):
    """x [*, d] with a share p of its entries (to the nearest 2^-16) zero and the others
    divided by the share that is kept.  Which ones is a function of the seed (an int, or
    an int64 tensor of one element on the device, read when the kernel runs), of the
    site, and of the entry's place: its row, counted from row0, and feature."""
    return _dropped(x, p, seed, site, row0, "x")


def dropout_bwd(dy, p: float, seed, site: int = 0, row0: int = 0):
    """The gradient of dropout_fwd: the same entries of dy."""
    return _dropped(dy, p, seed, site, row0, "dy")


class _DropoutFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, site, row0):
        ctx.seed = None if isinstance(seed, torch.Tensor) else seed
        ctx.save_for_backward(*([seed] if ctx.seed is None else []))  # (a seed that has changed since is an error)
        ctx.rest = (p, site, row0)
        return dropout_fwd(x, p, seed, site, row0)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        p, site, row0 = ctx.rest
        seed = ctx.saved_tensors[0] if ctx.seed is None else ctx.seed
        return dropout_bwd(dy.contiguous(), p, seed, site, row0), None, None, None, None


def dropout(x, p: float, seed, site: int = 0, row0: int = 0):
    """dropout_fwd's out; differentiable with respect to x."""
    return _DropoutFn.apply(x, p, seed, site, row0)


# -------------------------------------------------------------- residual norms

_VECTORS = ("gate", "post_w", "post_b", "pre_w", "pre_b")
_NAMES = ("x", "y", *_VECTORS)


class AddNormKept:
    """What add_norm_bwd needs of a call: its inputs, its options and four numbers a row."""

    __slots__ = ("x", "y", "vectors", "stats", "options")

    def __init__(self, x, y, vectors, stats, options):
        self.x, self.y, self.vectors, self.stats, self.options = x, y, vectors, stats, options


def _norm_call(x, y, vectors, options):
    """Checks the arguments; (device, infcl_add_norm)."""
    norm, eps, alpha, p, seed, site, row0 = options
    dev = _where(_NAMES, (x, y, *vectors))
    n, d, xs = _rows(x, "x")
    ys = 0
    gate, post_w, post_b, pre_w, pre_b = vectors
    if y is not None:
        if y.shape != x.shape or y.dtype != x.dtype:
            raise ValueError(f"y must be {tuple(x.shape)} of {x.dtype}, got {tuple(y.shape)} of {y.dtype}")
        ys = _rows(y, "y")[2]
    elif gate is not None or post_w is not None or p > 0 or alpha != 1:
        raise ValueError("gate, post_w, p and alpha come with y")
    elif pre_w is None:
        raise ValueError("there must be y or pre_w")
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {list(NORMS)}, got {norm!r}")
    if post_b is not None and post_w is None or pre_b is not None and pre_w is None:
        raise ValueError("a norm's bias comes with its weight")
    wdtype, dtype, ptrs = None, x.dtype, []
    for t in vectors:
        if t is None:
            ptrs.append(None)
            continue
        if t.dtype is not wdtype and (wdtype is not None or t.dtype not in (torch.float32, dtype)) or t.shape != (d,) or not t.is_contiguous():
            _wrong_vector(vectors, d, dtype)
        wdtype = t.dtype
        ptrs.append(t.data_ptr())
    code = _code(x, "x")
    return dev, _AddNorm(n, d, code, code if wdtype is None else _CODES[wdtype], NORMS[norm], eps, alpha,
                         _drop(p, seed, site, row0, dev), xs, ys, *ptrs)


def _wrong_vector(vectors, d, dtype):
    for k, t in zip(_VECTORS, vectors):
        if t is not None and (t.shape != (d,) or not t.is_contiguous() or t.dtype not in (torch.float32, dtype)):
            raise ValueError(f"{k} must be contiguous [{d}] of float32 or {dtype}, got {t.dtype} {tuple(t.shape)}")
    raise ValueError(f"gate and the norms' vectors must be of one dtype, got {[t.dtype for t in vectors if t is not None]}")


def add_norm_fwd(x, y=None, gate=None, post_w=None, post_b=None, pre_w=None, pre_b=None, norm: str = "layer",
                 eps: float = 1e-5, alpha: float = 1.0, p: float = 0.0, seed=0, site: int = 0, row0: int = 0,
                 need_grad: bool = True):
    """The residual sum after a block and the norm before the next one:

        t = y;  t = N(t) post_w + post_b;  t = dropout(t, p, seed, site, row0);  t = gate t
        h = alpha x + t;  z = N(h) pre_w + pre_b

    x, y [*, d]; gate and the norms' vectors [d], float32 or x's dtype.  What is not given
    is left out (without y: h = x; without pre_w: z is None).  norm: "layer" or "rms".
    Returns (h, z, kept), kept for add_norm_bwd (None without need_grad)."""
    vectors, options = (gate, post_w, post_b, pre_w, pre_b), (norm, float(eps), float(alpha), float(p), seed, site, row0)
    dev, a = _norm_call(x, y, vectors, options)
    h = x if y is None else _like(x)
    z = None if pre_w is None else _like(x)
    stats = torch.empty((a.n, 4), dtype=torch.float32, device=dev) if need_grad else None
    _call("infcl_add_norm_fwd", dev, ctypes.byref(a), x.data_ptr(), _ptr(y), _ptr(None if y is None else h), _ptr(z), _ptr(stats))
    return h, z, AddNormKept(x, y, vectors, stats, options) if need_grad else None


@functools.lru_cache(maxsize=4096)
def _norm_bytes(n, d):
    """Bytes of the backward's workspace, which rows and features alone decide."""
    a, size = _AddNorm(n, d, 0, 0, 0, 0.0, 1.0, _Drop(), d, d), ctypes.c_size_t(0)
    _check(_load().infcl_add_norm_bwd_workspace(ctypes.byref(a), ctypes.byref(size)), "infcl_add_norm_bwd_workspace")
    return size.value


def add_norm_bwd(dh, dz, kept: AddNormKept, need=(True,) * 7):
    """Gradients from those of h and z (None: zeros): (dx, dy, dgate, dpost_w, dpost_b,
    dpre_w, dpre_b), None for what was not given or is not needed.  Without y, dx counts
    z alone and dh where it is given."""
    x, y, vectors = kept.x, kept.y, kept.vectors
    dev, a = _norm_call(x, y, vectors, kept.options)
    if kept.stats.shape != (a.n, 4) or kept.stats.dtype != torch.float32 or not kept.stats.is_contiguous():
        raise ValueError(f"the kept statistics must be contiguous float32 [{a.n}, 4], got {tuple(kept.stats.shape)}")
    if dz is not None and vectors[3] is None:
        raise ValueError("there is no z without pre_w")
    strides = [0, 0]
    for i, (name, t) in enumerate((("dh", dh), ("dz", dz))):
        if t is not None:
            _where(("x", name), (x, t))
            if t.shape != x.shape or t.dtype != x.dtype:
                raise ValueError(f"{name} must be {tuple(x.shape)} of {x.dtype}, got {tuple(t.shape)} of {t.dtype}")
            strides[i] = _rows(t, name)[2]
    grads = [_like(x) if t is not None and w else None for t, w in zip((x, y), need)]
    grads += [torch.empty_like(t) if t is not None and w else None for t, w in zip(vectors, need[2:])]
    size = _norm_bytes(a.n, a.d)
    ws = _scratch(size, dev)
    g = _AddNormGrads(_ptr(dh), _ptr(dz), *strides, *(_ptr(t) for t in grads))
    _call("infcl_add_norm_bwd", dev, ctypes.byref(a), x.data_ptr(), _ptr(y), kept.stats.data_ptr(), ctypes.byref(g),
          ws.data_ptr(), size)
    return tuple(grads)


class _AddNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, grads, options, seed, x, y, *vectors):
        norm, eps, alpha, p, site, row0 = options
        learns = grads and any(ctx.needs_input_grad)
        h, z, kept = add_norm_fwd(x, y, *vectors, norm=norm, eps=eps, alpha=alpha, p=p, seed=seed, site=site, row0=row0,
                                  need_grad=learns)
        if learns:
            tensor = isinstance(seed, torch.Tensor)
            ctx.save_for_backward(x, y, *vectors, kept.stats, seed if tensor else None)
            ctx.options = (*options[:4], None if tensor else seed, *options[4:])
        ctx.set_materialize_grads(False)
        ctx.both = y is not None and z is not None
        return (h, z) if ctx.both else h if z is None else z

    @staticmethod
    @once_differentiable
    def backward(ctx, *d):
        x, y, *vectors, stats, seed = ctx.saved_tensors
        dh, dz = d if ctx.both else (d[0], None) if vectors[3] is None else (None, d[0])
        if dh is None and dz is None:
            return (None,) * 10
        options = ctx.options if seed is None else (*ctx.options[:4], seed, *ctx.options[5:])
        dh, dz = (t if t is None else t.contiguous() for t in (dh, dz))
        kept = AddNormKept(x, y, tuple(vectors), stats, options)
        return (None, None, None, *add_norm_bwd(dh, dz, kept, ctx.needs_input_grad[3:]))


def add_norm(x, y=None, gate=None, post_w=None, post_b=None, pre_w=None, pre_b=None, norm: str = "layer",
             eps: float = 1e-5, alpha: float = 1.0, p: float = 0.0, seed=0, site: int = 0, row0: int = 0):
    """add_norm_fwd's (h, z); differentiable with respect to x, y, gate and the norms'
    vectors."""
    args = (x, y, gate, post_w, post_b, pre_w, pre_b)
    res = _AddNormFn.apply(torch.is_grad_enabled(), (norm, float(eps), float(alpha), float(p), site, row0), seed, *args)
    return (x, res) if y is None else (res, None) if pre_w is None else res


# ---------------------------------------------------------------- 8-bit floats

class Fp8:
    """Rows [rows, k] in 8-bit floats: q [rows, 128 ceil(k / 128)] uint8 (E4M3 bytes; 128
    more where that is a multiple of 16384), exps [rows, 4 ceil(k / 512)] uint8 (a power of
    two for 128 entries), and the dtype they had."""

    __slots__ = ("q", "exps", "k", "dtype")

    def __init__(self, q, exps, k, dtype):
        self.q, self.exps, self.k, self.dtype = q, exps, k, dtype

    @property
    def shape(self):
        return (self.q.shape[0], self.k)

    def nbytes(self):
        return self.q.numel() + self.exps.numel()


def _fp8_widths(k):
    """Bytes of a row of values and of exponents."""
    kp = (k + BLOCK - 1) // BLOCK * BLOCK
    return kp + (BLOCK if kp and kp % 16384 == 0 else 0), (k + 511) // 512 * 4


def _fp8_room(rows, k, dtype, dev):
    kp, ep = _fp8_widths(k)
    return Fp8(torch.empty((rows, kp), dtype=torch.uint8, device=dev), torch.empty((rows, ep), dtype=torch.uint8, device=dev),
               k, dtype)


def _check_fp8(f, name):
    kp, ep = _fp8_widths(f.k)
    if f.q.dtype != torch.uint8 or f.exps.dtype != torch.uint8 or not f.q.is_contiguous() or not f.exps.is_contiguous():
        raise ValueError(f"{name} must hold contiguous uint8 values and exponents")
    if f.q.dim() != 2 or f.q.shape[1] != kp or f.exps.shape != (f.q.shape[0], ep):
        raise ValueError(f"{name}: values {tuple(f.q.shape)} and exponents {tuple(f.exps.shape)} do not fit rows of {f.k}")


def _fp8_pack(x, along=True, across=False, sums=False, name="x"):
    dev, code = _where((name,), (x,)), _code(x, name)
    n, d, stride = _rows(x, name)
    a = _fp8_room(n, d, x.dtype, dev) if along else None
    t = _fp8_room(d, n, x.dtype, dev) if across else None
    total = torch.empty(d, dtype=x.dtype, device=dev) if sums else None
    size = _bytes("infcl_fp8_pack_workspace", n, d) if sums else 0
    ws = _scratch(size, dev)
    if n or sums:
        _call("infcl_fp8_pack", dev, x.data_ptr(), stride, n, d, code, a.q.data_ptr() if a else None,
              a.exps.data_ptr() if a else None, t.q.data_ptr() if t else None, t.exps.data_ptr() if t else None,
              _ptr(total), _ptr(ws), size)
    return a, t, total


def fp8_pack(x) -> Fp8:
    """x [*, d] as rows of 8-bit floats with a power of two for every 128 features."""
    return _fp8_pack(x)[0]


def fp8_pack_both(x):
    """(fp8_pack of x [*, d], fp8_pack of its transpose [d, rows]) in one pass."""
    return _fp8_pack(x, True, True)[:2]


def fp8_unpack(f: Fp8):
    """What the 8-bit floats stand for, [rows, k] in the dtype x had."""
    _check_fp8(f, "the operand")
    dev = _device(("values", f.q), ("exponents", f.exps))
    out = torch.empty(f.shape, dtype=f.dtype, device=dev)
    _call("infcl_fp8_unpack", dev, f.q.data_ptr(), f.exps.data_ptr(), f.shape[0], f.k, _CODES[f.dtype], out.data_ptr())
    return out


def _out16(dtype, bias, m):
    """Checks what a product comes in; the bias as the kernels take it."""
    if dtype not in (torch.bfloat16, torch.float16):
        raise TypeError(f"products of 8-bit floats come in bfloat16 or float16, got {dtype}")
    if bias is None:
        return None
    if bias.shape != (m,) or bias.dtype != dtype or not bias.is_contiguous():
        raise ValueError(f"the bias must be contiguous [{m}] of {dtype}, got {bias.dtype} {tuple(bias.shape)}")
    return bias if bias.data_ptr() % 4 == 0 else bias.clone()  # (a view may begin at an odd entry)


def fp8_matmul(a: Fp8, b: Fp8, bias=None, dtype=None):
    """a b^T + bias, [rows of a, rows of b] in dtype (a's by default; bfloat16 or float16)."""
    _check_fp8(a, "a")
    _check_fp8(b, "b")
    dev = _where(("a", "a's exponents", "b", "b's exponents", "bias"), (a.q, a.exps, b.q, b.exps, bias))
    (n, k), (m, bk) = a.shape, b.shape
    if k != bk:
        raise ValueError(f"a and b must have rows of one length, got {k} and {bk}")
    dtype = a.dtype if dtype is None else dtype
    bias = _out16(dtype, bias, m)
    out = torch.empty((n, m), dtype=dtype, device=dev)
    if out.numel() == 0:
        return out
    size = _bytes("infcl_fp8_matmul_workspace", n, m, k)
    ws = _scratch(size, dev)
    _call("infcl_fp8_matmul", dev, a.q.data_ptr(), a.exps.data_ptr(), n, b.q.data_ptr(), b.exps.data_ptr(), m, k,
          _ptr(bias), _CODES[dtype], out.data_ptr(), _ptr(ws), size)
    return out


@functools.lru_cache(maxsize=4096)
def _layer_sizes(n, k, m, keeps):
    """Bytes of what is kept, of the forward's and of the backward's workspace."""
    sizes = [ctypes.c_size_t(0) for _ in range(3)]
    _check(_load().infcl_fp8_layer_sizes(n, k, m, keeps, *(ctypes.byref(s) for s in sizes)), "infcl_fp8_layer_sizes")
    return tuple(s.value for s in sizes)


_MOST_OUT = 1 << 23  # outputs of a layer with gradients


def _learns(m):
    if m % 8 or m > _MOST_OUT:
        raise ValueError(f"linear_fp8: a layer with gradients has a multiple of 8 outputs, up to 2^23, got {m}")


def linear_fp8_fwd(x, w, b=None, need_dx: bool = True, need_dw: bool = True):
    """(x w^T + b from x and w in 8-bit floats, what linear_fp8_bwd needs: both packed the
    other way round, where asked for).  x [*, k], w [m, k], b [m] of one 16-bit dtype."""
    dev, code = _where(("x", "w", "b"), (x, w, b)), _code(x, "x")
    if w.dim() != 2 or w.shape[1] != x.shape[-1] or w.dtype != x.dtype:
        raise ValueError(f"w must be [m, {x.shape[-1]}] of {x.dtype}, got {tuple(w.shape)} of {w.dtype}")
    (n, k, xs), (m, _, ws) = _rows(x, "x"), _rows(w, "w")
    b = _out16(x.dtype, b, m)
    keeps = need_dx + 2 * need_dw
    if keeps:
        _learns(m)
    elif m % 8 or m > _MOST_OUT:  # (a forward alone takes any number of outputs)
        return _times_packed(x, fp8_pack(w), b), (None, (n, k, m, x.dtype, 0, b is not None))
    size, scratch, _ = _layer_sizes(n, k, m, keeps)
    out = x.new_empty((*x.shape[:-1], m))
    kept, space = _scratch(size, dev), _scratch(scratch, dev)
    _call("infcl_fp8_layer_fwd", dev, x.data_ptr(), xs, n, k, w.data_ptr(), ws, m, _ptr(b), code, keeps, out.data_ptr(),
          _ptr(kept), space.data_ptr(), scratch)
    return out, (kept, (n, k, m, x.dtype, keeps, b is not None))


def linear_fp8_bwd(dy, kept, need=(True, True, True)):
    """(dx, dw, db) of linear_fp8_fwd, None where not kept for or not needed: products of
    dy in 8-bit floats, along its features for dx and along its rows for dw, and its sums."""
    kept, (n, k, m, dtype, keeps, has_b) = kept
    dev = _where(("dy", "what was kept"), (dy, kept))
    rows, width, stride = _rows(dy, "dy")
    if (rows, width, dy.dtype) != (n, m, dtype):
        raise ValueError(f"dy must be [{n}, {m}] of {dtype}, got {tuple(dy.shape)} of {dy.dtype}")
    size, _, scratch = _layer_sizes(n, k, m, keeps)
    if keeps and (kept.dtype != torch.uint8 or kept.numel() != size):
        raise ValueError(f"what was kept must be {size} bytes, got {kept.numel()} of {kept.dtype}")
    dx = torch.empty((*dy.shape[:-1], k), dtype=dtype, device=dev) if need[0] and keeps & 1 else None
    dw = torch.empty((m, k), dtype=dtype, device=dev) if need[1] and keeps & 2 else None
    db = torch.empty(m, dtype=dtype, device=dev) if need[2] and has_b else None
    if dx is not None or dw is not None or db is not None:
        space = _scratch(scratch, dev)
        _call("infcl_fp8_layer_bwd", dev, dy.data_ptr(), stride, n, k, m, _CODES[dtype], keeps, _ptr(kept), _ptr(dx), _ptr(dw),
              _ptr(db), space.data_ptr(), scratch)
    return dx, dw, db


class _LinearFp8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, grads, x, w, b):
        need_dx, need_dw = (grads and n for n in ctx.needs_input_grad[1:3])
        y, (kept, ctx.rest) = linear_fp8_fwd(x, w, b, need_dx, need_dw)
        ctx.save_for_backward(kept)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        return (None, *linear_fp8_bwd(dy.contiguous(), (ctx.saved_tensors[0], ctx.rest), ctx.needs_input_grad[1:]))


class _LinearPacked(torch.autograd.Function):
    """The forward alone, for a trace to record and forward mode to refuse."""

    @staticmethod
    def forward(ctx, x, q, exps, k, dtype, b):
        return _times_packed(x, Fp8(q, exps, k, dtype), b)


def linear_fp8(x, w, b=None):
    """x w^T + b with products of 8-bit floats (a power of two for each 128 entries of
    the contraction), forward and both gradients; between the passes it keeps x and w in 8
    bits.  x [*, k] and w [m, k] (k a multiple of 8; m too where there are gradients), b [m] of
    one 16-bit dtype, or of any under autocast.  w may be an Fp8 of the weights, packed
    once: the forward alone, up to 16 rows in one launch."""
    if isinstance(w, Fp8):
        return _linear_packed(x, w, b)
    if torch.is_autocast_enabled("cuda"):
        dtype = torch.get_autocast_dtype("cuda")
        x, w, b = x.to(dtype), w.to(dtype), None if b is None else b.to(dtype)
    grads = torch.is_grad_enabled()
    if grads and any(t is not None and t.requires_grad for t in (x, w, b)):
        _learns(w.shape[0])
    return _LinearFp8.apply(grads, x, w, b)


def _linear_packed(x, w, b):
    if torch.is_grad_enabled() and (x.requires_grad or b is not None and b.requires_grad):
        raise ValueError("a layer of packed weights has no backward pass: call it under no_grad, or give the weights")
    _check_fp8(w, "w")
    if torch.is_autocast_enabled("cuda"):
        x = x.to(torch.get_autocast_dtype("cuda"))
        b = None if b is None else b.to(x.dtype)
    if forward_ad._current_level < 0 and not torch.jit.is_tracing():  # (2.5 us less a call)
        return _times_packed(x, w, b)
    return _LinearPacked.apply(x, w.q, w.exps, w.k, w.dtype, b)


def _times_packed(x, w, b):
    dev = _where(("x", "w", "w's exponents", "b"), (x, w.q, w.exps, b))
    n, k, stride = _rows(x, "x")
    m = w.shape[0]
    if k != w.k:
        raise ValueError(f"x must have rows of {w.k}, got {tuple(x.shape)}")
    b = _out16(x.dtype, b, m)
    out = x.new_empty((*x.shape[:-1], m))
    if out.numel() == 0:
        return out
    size = _bytes("infcl_fp8_linear_workspace", n, m, k)
    ws = _scratch(size, dev)
    _call("infcl_fp8_linear", dev, x.data_ptr(), stride, n, k, w.q.data_ptr(), w.exps.data_ptr(), m, _ptr(b),
          _CODES[x.dtype], out.data_ptr(), _ptr(ws), size)
    return out
