"""Binding of include/acp_ops.h: the operators around the attention of `acp`.

  layer_norm, rms_norm      differentiable norms; norm_forward / norm_backward without autograd
  Rotary                    rotary positions of queries and keys
  PagedCache                a cache of many sequences in pages of 64 positions, and the
                            attention of new tokens over it

Argument marshalling only, as in `acp`: every step runs in the library's kernels, on
PyTorch's current stream of the tensors' device.  A serving step of a QK-normed layer:

    q, k = ops.rms_norm(q, wq), ops.rms_norm(k, wk)            # [1, H, T, d], w [H, d]
    q, k = rope(q, k, positions)                               # positions [T]
    cache.append(k[0].transpose(0, 1), v, log_f, cu, past, table)
    o, lse = cache.attend(q[0].transpose(0, 1), cu, past, table, max_new,
                          gamma_q=gq, gamma_k=gk, eps=eps, L_max=L_max)

and of training: rms_norm, rope, then acp.fox_attention.  Into a HIP graph record the calls
without autograd (norm_forward, norm_backward, Rotary.forward and backward, append, attend): a
backward() recorded while an eager graph of the same leaves is alive works on that graph's
stream, which can end the process.
"""
from __future__ import annotations

import ctypes
import math
import os
import re

import torch
from torch.autograd.function import once_differentiable

from . import acp
from .acp import ACP_BF16, ACP_F32, AcpError

HEADER = os.path.join(os.path.dirname(acp.HEADER), "acp_ops.h")

PAGE = 64                    # positions per page
FLAG_BAD_PAGE = 64
FLAG_MAX_NEW = 128
FLAG_SCALES = 256

OP_NAMES = ("norm", "norm_bwd", "rotary", "append", "attend")
_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "ramp": 3}


class PagedLayout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("k", "v", "c", "total")]


class OpTimes(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_int64 * len(OP_NAMES)), ("ms", ctypes.c_double * len(OP_NAMES))]


_i, _d, _p, _sz, _i64 = (ctypes.c_int, ctypes.c_double, ctypes.c_void_p, ctypes.c_size_t,
                         ctypes.c_int64)
_SIGS = {
    "acp_norm_fwd": [_p, _p, _p, _p] + [_i] * 8 + [_d, _p, _p, _p, _p],
    "acp_norm_workspace_size": [_i] * 5 + [ctypes.POINTER(_sz)],
    "acp_norm_bwd": [_p] * 5 + [_i] * 7 + [_p] * 7 + [_sz, _p],
    "acp_rotary_table": [_i, _d, _i, _d, _d, _d, _d, ctypes.POINTER(_d)],
    "acp_rotary": [_p] * 4 + [_i] * 9 + [_d, _p, _p, _i, _p, _i64] + [_p] * 5,
    "acp_paged_cache_size": [_i] * 5 + [ctypes.POINTER(_sz)],
    "acp_paged_offsets": [_i] * 5 + [ctypes.POINTER(PagedLayout)],
    "acp_paged_append": [_p] * 6 + [_i] * 8 + [_p] * 4 + [_sz, _p, _p],
    "acp_paged_workspace_size": [_i] * 7 + [_i64, ctypes.POINTER(_sz)],
    "fox_attn_paged": ([_p] * 2 + [_i] * 8 + [_p] * 4 + [_sz, _p, _p, _d, _i64, _i, _i64] + [_p] * 4
                       + [_sz, _p]),
    "acp_op_timing_read": [ctypes.POINTER(OpTimes)],
}
_SIGS["fox_attn_paged_filled"] = _SIGS["fox_attn_paged"]
_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = acp.lib()
        for name, args in _SIGS.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = _i
        _lib = L
    return _lib


def header_functions() -> list:
    """Names of the functions include/acp_ops.h declares."""
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return re.findall(r"^\s*(?:const\s+)?\w+\*?\s+\*?(\w+)\s*\(", text, flags=re.M)


def acp_op_timing_read() -> dict:
    """{operator: (calls, summed ms)} since acp.acp_timing_reset() (waits for the GPU)."""
    t = OpTimes()
    acp._check(lib().acp_op_timing_read(ctypes.byref(t)))
    return {n: (int(t.launches[i]), float(t.ms[i])) for i, n in enumerate(OP_NAMES)}


# ---- marshalling -----------------------------------------------------------------------

def _device(*ts):
    """The device of all of them, by index (cheaper than device objects)."""
    d = ts[0].get_device()
    for t in ts:
        if t.get_device() != d:
            raise ValueError("tensors must live on one GPU")
    if d < 0:
        raise ValueError("tensors must live on the GPU")
    return d


def _stream(d: int) -> int:
    if acp._raw_stream is not None:
        return acp._raw_stream(d)
    return torch.cuda.current_stream(d).cuda_stream


def _run(fn, d, *args):
    """fn(*args, stream) on the current stream of device d."""
    if d == torch.cuda.current_device():
        status = fn(*args, _stream(d))
    else:
        with torch.cuda.device(d):
            status = fn(*args, _stream(d))
    if status != acp.ACP_OK:
        acp._check(status)


def _strides(t: torch.Tensor):
    """Element strides of the three leading axes of a 4-D tensor (None: contiguous)."""
    if t.is_contiguous():
        return None
    s = t.stride()
    return (_i64 * 3)(s[0], s[1], s[2])


def _contiguous_like(t: torch.Tensor) -> torch.Tensor:
    """An empty contiguous tensor like t (empty_like where it is one: 0.6 us less than new_empty)."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---- norms -----------------------------------------------------------------------------

def _rows(x: torch.Tensor, weight: torch.Tensor):
    """(x as [B, H, L, n] with contiguous features, per_head) for a weight [n] or [H, n]."""
    if x.dim() < 1 or weight.shape[-1] != x.shape[-1]:
        raise ValueError("weight must match x's last axis")
    if x.stride(-1) != 1 and x.shape[-1] > 1:
        x = x.contiguous()
    if weight.dim() == 2:
        if x.dim() != 4 or weight.shape[0] != x.shape[1]:
            raise ValueError("a weight [H, n] needs x [B, H, L, n]")
        return x, True
    if weight.dim() != 1:
        raise ValueError("weight must be [n] or [H, n]")
    if x.dim() == 4:
        return x, False
    if x.is_contiguous() or x.dim() > 4:
        return x.contiguous().view(1, 1, -1 if x.numel() else 0, x.shape[-1]), False
    return x.reshape((1,) * (4 - x.dim()) + x.shape), False


def _check_weight(name, t, weight):
    if t is not None and (t.shape != weight.shape or t.dtype != weight.dtype):
        raise ValueError(name + " must match weight")


def norm_forward(x, weight, bias=None, eps: float = 1e-6, center: bool = False, stats: bool = True,
                 out=None):
    """(y, mean, rstd) of acp_norm_fwd: y like x (contiguous), mean (None without
    `center`) and rstd float32 of x's leading axes, or None without `stats`.

    x [..., n] float32 or bfloat16, of any strides along the leading axes; weight (and
    bias) [n], or [H, n] for x [B, H, L, n], float32 or bfloat16, contiguous."""
    dev = _device(x, weight) if bias is None else _device(x, weight, bias)
    x4, per_head = _rows(x, weight)
    _check_weight("bias", bias, weight)
    if not weight.is_contiguous() or (bias is not None and not bias.is_contiguous()):
        raise ValueError("weight and bias must be contiguous")
    B, H, L, n = x4.shape
    y = _contiguous_like(x) if out is None else out
    if out is not None and (out.shape != x.shape or out.dtype != x.dtype or not out.is_contiguous()
                            or out.get_device() != dev):
        raise ValueError("out must be contiguous and like x")
    mean = x.new_empty(x.shape[:-1], dtype=torch.float32) if stats and center else None
    rstd = x.new_empty(x.shape[:-1], dtype=torch.float32) if stats else None
    _run(lib().acp_norm_fwd, dev, x4.data_ptr(), _strides(x4), weight.data_ptr(), _ptr(bias), acp._dt(x),
         acp._dt(weight), B, H, L, n, per_head, center, eps, y.data_ptr(), _ptr(mean), _ptr(rstd))
    return y, mean, rstd


def norm_backward(dy, x, weight, mean, rstd, bias: bool = False):
    """(dx, dweight, dbias) for norm_forward's inputs and statistics; dx has x's strides
    where x is dense, dweight and dbias (None without `bias`) are float32."""
    dev = _device(dy, x, weight, rstd)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must match x")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t is not None and (t.shape != x.shape[:-1] or t.dtype != torch.float32
                              or not t.is_contiguous() or t.get_device() != dev):
            raise ValueError(name + " must be norm_forward's")
    if not weight.is_contiguous():
        raise ValueError("weight must be contiguous")
    x4, per_head = _rows(x, weight)
    dy4 = dy
    if dy.stride(-1) != 1 and dy.shape[-1] > 1 or (dy.dim() != 4 and not dy.is_contiguous()):
        dy4 = dy.contiguous()
    B, H, L, n = x4.shape
    dy4 = dy4.view(x4.shape) if dy4.dim() != 4 else dy4
    dx4 = torch.empty_like(x4)
    if dx4.stride(3) != 1 and n > 1:         # (x's rows share features: no order of the axes to take over)
        dx4 = x4.new_empty(x4.shape)
    dw = x.new_empty(weight.shape, dtype=torch.float32)
    db = torch.empty_like(dw) if bias else None
    need = _sz(0)
    acp._check(lib().acp_norm_workspace_size(B, H, L, n, per_head, ctypes.byref(need)))
    ws = dw.new_empty(need.value // 4 + 4)
    _run(lib().acp_norm_bwd, dev, dy4.data_ptr(), _strides(dy4), x4.data_ptr(), _strides(x4),
         weight.data_ptr(), acp._dt(x), acp._dt(weight), B, H, L, n, per_head, _ptr(mean), rstd.data_ptr(),
         dx4.data_ptr(), _strides(dx4), dw.data_ptr(), _ptr(db), ws.data_ptr(), 4 * ws.numel())
    return dx4.view(x.shape) if dx4.shape != x.shape else dx4, dw, db


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, center):
        y, mean, rstd = norm_forward(x, weight, bias, eps, center, stats=any(ctx.needs_input_grad))
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.has_bias = bias is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = norm_backward(dy.to(x.dtype), x, weight, mean, rstd, ctx.has_bias)
        return dx, dw.to(weight.dtype), None if db is None else db.to(weight.dtype), None, None


def layer_norm(x, weight, bias=None, eps: float = 1e-5):
    """Differentiable layer norm over x's last axis (see norm_forward for the arguments)."""
    return _Norm.apply(x, weight, bias, eps, True)


def rms_norm(x, weight, eps: float = 1e-6):
    """Differentiable RMS norm over x's last axis; with x [B, H, L, d] and weight [H, d]
    the QK-norm, whose gamma (acp.forward_qknorm, PagedCache.attend) is weight.abs().amax(-1)."""
    return _Norm.apply(x, weight, None, eps, False)


# ---- rotary positions --------------------------------------------------------------------

class Rotary:
    """Rotary positions for the first `rot` features of a head.

    layout   "half": pairs (i, i + rot/2); "interleaved": pairs (2 i, 2 i + 1)
    scaling  for contexts `factor` times as long: "none", "linear", "base" or "ramp" (by
             the turns a pair makes over `train_len`, from `slow` to `fast`); see acp_ops.h
    amplitude multiplies the turned features; by default 1, and 0.1 ln(factor) + 1 with
             "ramp" (the attention's logits then grow by its square, and so does the
             bound that QK-norm scales give: enlarge gamma by it)
    """

    def __init__(self, rot: int, base: float = 10000.0, layout: str = "half", scaling: str = "none",
                 factor: float = 1.0, train_len: float = 0.0, slow: float = 1.0, fast: float = 32.0,
                 amplitude: float | None = None, device="cuda"):
        if layout not in _LAYOUTS or scaling not in _SCALINGS:
            raise ValueError("unknown layout or scaling")
        self.rot, self.layout = rot, _LAYOUTS[layout]
        table = (_d * max(rot // 2, 1))()
        acp._check(lib().acp_rotary_table(rot, base, _SCALINGS[scaling], factor, train_len, slow, fast, table))
        self.turns = torch.tensor(list(table), dtype=torch.float64).to(device)
        if amplitude is None:
            amplitude = 0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0
        self.amplitude = amplitude

    def forward(self, q, k=None, positions=None, start: int = 0, out=None):
        """(q, k) turned, without autograd.  q [B, H, L, d] and k [B, Hk, L, d], of any
        strides with contiguous features; positions [L] or [B, L] int32 or int64, or
        position l is start + l.  out: (q_out, k_out), which may be the inputs."""
        return self._turn(q, k, positions, start, out, 0)

    def backward(self, dq, dk=None, positions=None, start: int = 0, out=None):
        """Gradients of forward()'s inputs from those of its outputs."""
        return self._turn(dq, dk, positions, start, out, 1)

    def __call__(self, q, k=None, positions=None, start: int = 0):
        """Differentiable forward()."""
        return _Rotate.apply(q, k, self, positions, start)

    def _turn(self, q, k, positions, start, out, inverse):
        dev = _device(q, self.turns) if k is None else _device(q, k, self.turns)
        if q.dim() != 4 or (k is not None and (k.dim() != 4 or k.shape[0] != q.shape[0]
                                               or k.shape[2:] != q.shape[2:] or k.dtype != q.dtype)):
            raise ValueError("q must be [B, H, L, d] and k [B, Hk, L, d] of its type")
        B, H, L, d = q.shape
        if out is None:
            out = (_contiguous_like(q), None if k is None else _contiguous_like(k))
        for t, o in zip((q, k), out):
            if t is None:
                continue
            if t.stride(3) != 1 or o.stride(3) != 1:
                raise ValueError("features must be contiguous")
            if o.shape != t.shape or o.dtype != t.dtype or o.get_device() != dev:
                raise ValueError("out must be like its input")
        pos = None
        if positions is not None:
            if positions.dtype not in (torch.int32, torch.int64) or positions.get_device() != dev:
                raise ValueError("positions must be int32 or int64 on the tensors' GPU")
            if tuple(positions.shape) == (L,):
                pos = (_i64 * 2)(0, positions.stride(0))
            elif tuple(positions.shape) == (B, L):
                pos = (_i64 * 2)(positions.stride(0), positions.stride(1))
            else:
                raise ValueError("positions must be [L] or [B, L]")
        qo, ko = out
        _run(lib().acp_rotary, dev, q.data_ptr(), _strides(q), _ptr(k), None if k is None else _strides(k),
             acp._dt(q), B, H, 0 if k is None else k.shape[1], L, d, self.rot, self.layout, inverse,
             self.amplitude, self.turns.data_ptr(), _ptr(positions),
             0 if positions is None else positions.element_size(), pos, start, qo.data_ptr(), _strides(qo),
             _ptr(ko) if k is not None else None, None if k is None else _strides(ko))
        return qo, ko if k is not None else None


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, rope, positions, start):
        ctx.rope, ctx.start, ctx.two = rope, start, k is not None
        ctx.save_for_backward(positions)
        return rope.forward(_features(q), _features(k), positions, start)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        positions, = ctx.saved_tensors
        dq, dk = ctx.rope.backward(_features(dq), _features(dk) if ctx.two else None, positions, ctx.start)
        return dq, dk, None, None, None


def _features(t):
    return t if t is None or t.stride(3) == 1 else t.contiguous()


# ---- paged cache ---------------------------------------------------------------------------

class PagedCache:
    """`pages` pages of 64 positions for H query heads, Hk key heads of d features (64 or
    128; float32 or bfloat16): keys, values and cumulative gates in one device buffer.

    A call names its N sequences by int32 tensors: cu [N + 1] (sequence s brings the packed
    rows cu[s] .. cu[s + 1] - 1), past [N] (positions held before them) and table [N, W] (its
    pages).  Which pages are free is the caller's to know; acp_ops.h states what a page number
    out of range does and what `flags` ([N, H] int32, written if given) reports."""

    def __init__(self, pages: int, H: int, d: int, Hk: int | None = None, dtype=torch.bfloat16,
                 device="cuda"):
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("the cache holds float32 or bfloat16")
        self.P, self.H, self.d, self.Hk, self.dtype = pages, H, d, H if Hk is None else Hk, dtype
        self.dt = ACP_F32 if dtype == torch.float32 else ACP_BF16
        n = _sz(0)
        acp._check(lib().acp_paged_cache_size(pages, H, self.Hk, d, self.dt, ctypes.byref(n)))
        self.buffer = torch.empty(n.value, dtype=torch.uint8, device=device)
        y = PagedLayout()
        acp._check(lib().acp_paged_offsets(pages, H, self.Hk, d, self.dt, ctypes.byref(y)))
        kv = (pages, self.Hk, PAGE, d)
        self._views = {"k": self.buffer[y.k:y.v].view(dtype).view(kv),
                       "v": self.buffer[y.v:y.c].view(dtype).view(kv),
                       "c": self.buffer[y.c:y.total].view(torch.float64).view(pages, H, PAGE)}

    def views(self) -> dict:
        """Views of the pages: k, v [P, Hk, 64, d], c [P, H, 64] float64."""
        return dict(self._views)

    def _sequences(self, cu, past, table, flags):
        for name, t in (("cu", cu), ("past", past), ("table", table), ("flags", flags)):
            if t is not None and (t.dtype != torch.int32 or not t.is_contiguous()):
                raise ValueError(name + " must be contiguous int32")
        N = past.shape[0]
        if past.dim() != 1 or cu.shape != (N + 1,) or table.dim() != 2 or table.shape[0] != N:
            raise ValueError("cu must be [N + 1], past [N] and table [N, W]")
        if flags is not None and flags.shape != (N, self.H):
            raise ValueError("flags must be [N, H]")
        return N, table.shape[1]

    def _packed(self, name, t, heads):
        if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != self.d or t.dtype != self.dtype:
            raise ValueError(f"{name} must be [T, {heads}, {self.d}] of the cache's type")
        if t.stride(2) != 1:
            raise ValueError(name + ": features must be contiguous")
        # (an axis of one has any stride)
        if t.is_contiguous():
            return None
        return (_i64 * 2)(t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if heads > 1 else 0)

    def append(self, k, v, log_f, cu, past, table, flags=None):
        """Store new rows: k, v [T, Hk, d] (strided rows of 16-byte alignment), log_f [T, H] float32."""
        ts = (k, v, log_f, cu, past, table, self.buffer)
        dev = _device(*ts) if flags is None else _device(*ts, flags)
        N, W = self._sequences(cu, past, table, flags)
        T = k.shape[0]
        ks, vs = self._packed("k", k, self.Hk), self._packed("v", v, self.Hk)
        if v.shape[0] != T or log_f.shape != (T, self.H) or log_f.dtype != torch.float32:
            raise ValueError("v must be like k, and log_f float32 [T, H]")
        _run(lib().acp_paged_append, dev, k.data_ptr(), ks, v.data_ptr(), vs, log_f.data_ptr(),
             None if log_f.is_contiguous() else (_i64 * 2)(log_f.stride(0), log_f.stride(1)), self.dt, T, N, W,
             self.P, self.H, self.Hk, self.d, cu.data_ptr(), past.data_ptr(), table.data_ptr(),
             self.buffer.data_ptr(), self.buffer.numel(), _ptr(flags))

    def attend(self, q, cu, past, table, max_new: int, max_len: int | None = None, gamma_q=None,
               gamma_k=None, eps: float = 0.0, L_max: int = 131072, out=None, flags=None):
        """(O [T, H, d], lse [T, H]) of the new rows q [T, H, d], after append() of the same
        rows.  max_new bounds a sequence's new rows; max_len (by default the table's, at most 2^31)
        its length, as a hint.  Rows from cu[N] on, and those of a sequence with more than max_new
        (flags reports it) that are not attended for, get O = 0 and lse = -inf; in `out` they stay
        as they are.
        eps > 0 prunes with gamma_q [H], gamma_k [Hk] float32, for sequences up to L_max.  The scales
        must bound the logits, |q.k| / sqrt(d) <= gamma_q gamma_k sqrt(d), as the largest |weight| of
        QK-normed rows does (times the square of a Rotary's amplitude above 1): they decide what is
        pruned, and keep the weights of bfloat16 chunks in range (flags reports FLAG_SCALES where they
        did not)."""
        ts = (q, cu, past, table, self.buffer)
        dev = _device(*ts) if flags is None else _device(*ts, flags)
        N, W = self._sequences(cu, past, table, flags)
        qs = self._packed("q", q, self.H)
        T = q.shape[0]
        if eps > 0.0:
            for name, t, heads in (("gamma_q", gamma_q, self.H), ("gamma_k", gamma_k, self.Hk)):
                if t is None or t.shape != (heads,) or t.dtype != torch.float32 or t.get_device() != dev \
                        or not t.is_contiguous():
                    raise ValueError(f"{name} must be float32 [{heads}]")
        else:
            gamma_q = gamma_k = None
        if out is None:
            o = _contiguous_like(q)
            lse = q.new_empty((T, self.H), dtype=torch.float32)
        else:
            o, lse = out
            if o.shape != (T, self.H, self.d) or o.dtype != self.dtype or lse.shape != (T, self.H) \
                    or lse.dtype != torch.float32 or not (o.is_contiguous() and lse.is_contiguous()) \
                    or o.get_device() != dev or lse.get_device() != dev:
                raise ValueError("out must be contiguous (O [T, H, d], lse [T, H])")
        if max_len is None:
            max_len = min(PAGE * W, 1 << 31)
        need = _sz(0)
        acp._check(lib().acp_paged_workspace_size(T, N, self.H, self.Hk, self.d, self.dt, max_new, max_len,
                                                  ctypes.byref(need)))
        ws = self.buffer.new_empty(need.value) if need.value else None
        fn = lib().fox_attn_paged_filled if out is None else lib().fox_attn_paged
        _run(fn, dev, q.data_ptr(), qs, self.dt, T, N, W, self.P, self.H, self.Hk, self.d, cu.data_ptr(),
             past.data_ptr(), table.data_ptr(), self.buffer.data_ptr(), self.buffer.numel(), _ptr(gamma_q),
             _ptr(gamma_k), eps, L_max, max_new, max_len, o.data_ptr(), lse.data_ptr(), _ptr(flags), _ptr(ws),
             need.value)
        return o, lse
