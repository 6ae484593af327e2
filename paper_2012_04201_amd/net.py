"""Operators of a wide residual network in 8 bits (the C ABI of include/bbo_net.h) on torch tensors.

    norm = net.rms_norm(x, weight, residual=r, want_8bit=True)        # norm.y8, norm.sum
    w8, w8t = net.quantize(weight, tile=128, want_cols=True)
    y = net.matmul8(norm.y8, w8)                                      # y = norm(x + r) weight^T
    opt = net.AdamW(params, lr=1e-3, state="8bit"); opt.step(grads)

Argument marshalling only, as in `binding`: every value is computed in the HIP kernels, PyTorch supplies device memory and
the stream.  Inputs are on the GPU; calls work on the current device's current stream, or on `stream`, and do not wait.
"""
import ctypes as C
import functools
from collections import namedtuple

import numpy as np
import torch

from . import binding
from .binding import BF16, F32, OK, BboError

EXPORTS = ["bbo_net_rms_norm", "bbo_net_rms_norm_grad_workspace", "bbo_net_rms_norm_grad", "bbo_net_quantize",
           "bbo_net_matmul8_workspace", "bbo_net_matmul8", "bbo_net_adamw", "bbo_net_last_error"]

BLOCK = 128
MOMENTS_F32, MOMENTS_8BIT = 0, 1

#: A matrix in 8 bits: values float8_e4m3fn [rows, cols], scales float8_e8m0fnu [ceil(rows / tile), ceil(cols / 128)].
Blocks8 = namedtuple("Blocks8", "values scales tile")
#: What rms_norm gives; None for what was not asked for.
Norm = namedtuple("Norm", "y sum rstd y8")
#: A tensor's moments in 8 bits: codes float8_e4m3fn like the tensor, scales float32 [ceil(n / 128)].
State8 = namedtuple("State8", "m m_scales v v_scales")

_P, _I64, _I32, _F, _U64, _SZ = C.c_void_p, C.c_int64, C.c_int32, C.c_float, C.c_uint64, C.c_size_t
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_E4M3, _E8M0, _FLOAT = torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.float32
_new = torch.empty_strided


class Tensor(C.Structure):
    _fields_ = [("p", _P), ("g", _P), ("m", _P), ("v", _P), ("m_scales", _P), ("v_scales", _P), ("copy", _P), ("n", _I64),
                ("lr", _F), ("weight_decay", _F)]


_net = None


def lib():
    """The shared library with these functions' argument types."""
    global _net
    if _net is None:
        L = binding.lib()
        L.bbo_net_last_error.restype = C.c_char_p
        L.bbo_net_rms_norm.argtypes = [_P, _I64, _P, _I64, _P, _I64, _I64, _F, _I32, _P, _I64, _P, _I64, _P, _P, _I64, _P, _I64, _P]
        L.bbo_net_rms_norm_grad_workspace.argtypes = [_I64, _I64, C.POINTER(_SZ)]
        L.bbo_net_rms_norm_grad.argtypes = [_P, _I64, _P, _I64, _P, _I64, _P, _P, _I64, _I64, _I32, _P, _I64, _P, _P, _SZ, _P]
        L.bbo_net_quantize.argtypes = [_P, _I64, _P, _I64, _I64, _I64, _I32, _I32, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P]
        L.bbo_net_matmul8_workspace.argtypes = [_I64, _I64, _I64, C.POINTER(_SZ)]
        L.bbo_net_matmul8.argtypes = [_P, _I64, _P, _I64, _I32, _P, _I64, _P, _I64, _I32, _I64, _I64, _I64, _P, _I64, _I32, _I32, _P, _SZ, _P]
        L.bbo_net_adamw.argtypes = [C.POINTER(Tensor), _I32, _I32, _I32, _I32, C.c_double, C.c_double, C.c_double, _I64, _U64, _P, _P]
        _net = L
    return _net


def _check(rc):
    if rc != OK:
        raise BboError(rc, lib().bbo_net_last_error().decode())


_current = torch._C._cuda_getCurrentRawStream  # of a device; torch.cuda.current_stream() takes 2.7 us to say the same


def _stream(stream, t):
    return _current(t.get_device()) if stream is None else stream.cuda_stream


def _room(stream, shape, stride, dtype, device):
    """A tensor for an output: under the stream that will use it."""
    if stream is None:
        return _new(shape, stride, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return _new(shape, stride, dtype=dtype, device=device)


def _matrix(t, name, like=None):
    """A [rows, cols] tensor on the GPU whose rows are dense; of another's type, shape and device."""
    shape = t.shape
    if len(shape) != 2 or (t.stride(1) != 1 and shape[1] > 1):
        raise ValueError("%s must be a [rows, cols] tensor with dense rows" % name)
    if like is None:
        if t.dtype not in _DTYPES:
            raise ValueError("%s must be float32 or bfloat16" % name)
        if not t.is_cuda:
            raise ValueError("%s must be on the GPU" % name)
    elif t.dtype is not like.dtype or shape != like.shape or t.get_device() != like.get_device():
        raise ValueError("%s must be %s %s on %s" % (name, like.dtype, tuple(like.shape), like.device))


def _row(t):
    """The distance of a matrix's rows: a single row's stride says nothing."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _vector(t, name, n, like):
    if t.dtype is not _FLOAT or t.shape != (n,) or not t.is_contiguous() or t.get_device() != like.get_device():
        raise ValueError("%s must be a dense float32 [%d] tensor on the same GPU" % (name, n))


def empty_blocks8(rows, cols, tile=1, device="cuda", stream=None):
    """Room for an 8-bit matrix: rows at multiples of 128 bytes, their scales at multiples of 4."""
    kb = (cols + 127) >> 7
    v = _room(stream, (rows, cols), (kb * BLOCK, 1), _E4M3, device)
    s = _room(stream, (rows if tile == 1 else (rows + 127) >> 7, kb), ((kb + 3) & ~3, 1), _E8M0, device)
    return Blocks8(v, s, tile)


def _check_blocks(b, name):
    v, s, tile = b
    if tile != 1 and tile != BLOCK:
        raise ValueError("%s: tile must be 1 or 128" % name)
    shape = v.shape
    if len(shape) != 2 or v.dtype is not _E4M3 or (v.stride(1) != 1 and shape[1] > 1):
        raise ValueError("%s: values must be float8_e4m3fn [rows, cols] with dense rows" % name)
    rows, cols = shape
    want = (rows if tile == 1 else (rows + 127) >> 7, (cols + 127) >> 7)
    if s.dtype is not _E8M0 or s.shape != want or (s.stride(1) != 1 and want[1] > 1):
        raise ValueError("%s: scales must be float8_e8m0fnu %s with dense rows" % (name, want))
    if not v.is_cuda or s.get_device() != v.get_device():
        raise ValueError("%s must be on the GPU" % name)
    return rows, cols


@functools.lru_cache(4096)
def _product_room(m, n, k):
    need = _SZ(0)
    _check(lib().bbo_net_matmul8_workspace(m, n, k, C.byref(need)))
    return need.value


@functools.lru_cache(4096)
def _grad_room(rows, width):
    need = _SZ(0)
    _check(lib().bbo_net_rms_norm_grad_workspace(rows, width, C.byref(need)))
    return max(need.value, 256)


def rms_norm(x, weight=None, residual=None, eps=1e-6, want_y=True, want_rstd=False, want_8bit=False, stream=None):
    """h = x + residual (kept as `sum`); y = h / sqrt(mean(h^2) + eps) * weight, per row of x [rows, width].

    weight: float32 [width] or None.  y has x's type; y8 is y in 8 bits (tile 1), rounded once.  rstd is for the gradient."""
    _matrix(x, "x")
    rows, width = x.shape
    dtype, device = x.dtype, x.device
    y = h = rstd = y8 = None
    pr = pw = ph = py = ps = 0
    r_stride, q = 0, (0, 0, 0, 0)
    if residual is not None:
        _matrix(residual, "residual", x)
        pr, r_stride = residual.data_ptr(), _row(residual)
        h = _room(stream, (rows, width), (width, 1), dtype, device)
        ph = h.data_ptr()
    if weight is not None:
        _vector(weight, "weight", width, x)
        pw = weight.data_ptr()
    if want_y:
        y = _room(stream, (rows, width), (width, 1), dtype, device)
        py = y.data_ptr()
    if want_rstd:
        rstd = _room(stream, (rows,), (1,), torch.float32, device)
        ps = rstd.data_ptr()
    if want_8bit:
        y8 = empty_blocks8(rows, width, 1, device, stream)
        q = (y8.values.data_ptr(), _row(y8.values), y8.scales.data_ptr(), _row(y8.scales))
    _check((_net or lib()).bbo_net_rms_norm(x.data_ptr(), _row(x), pr, r_stride, pw, rows, width, eps, _DTYPES[dtype], ph, width, py, width, ps, *q,
                                            _stream(stream, x)))
    return Norm(y, h, rstd, y8)


def rms_norm_grad(dy, h, rstd, weight=None, dsum=None, want_dweight=True, workspace=None, stream=None):
    """(dx, dweight) of rms_norm: h is its x, or its sum where it had a residual; dsum the gradient that arrives at sum.

    dx is the gradient of x and of residual alike; dweight (float32) is None if not wanted."""
    _matrix(h, "h")
    rows, width = h.shape
    dtype, device = h.dtype, h.device
    _matrix(dy, "dy", h)
    _vector(rstd, "rstd", rows, h)
    pd = pw = pg = ws = room = d_stride = 0
    if dsum is not None:
        _matrix(dsum, "dsum", h)
        pd, d_stride = dsum.data_ptr(), _row(dsum)
    if weight is not None:
        _vector(weight, "weight", width, h)
        pw = weight.data_ptr()
    dx, dw = _room(stream, (rows, width), (width, 1), dtype, device), None
    L = _net or lib()
    if want_dweight:
        dw = _room(stream, (width,), (1,), torch.float32, device)
        pg = dw.data_ptr()
        if workspace is None:
            workspace = _room(stream, (_grad_room(rows, width),), (1,), torch.uint8, device)
        elif workspace.device != device or not workspace.is_contiguous():
            raise ValueError("workspace must be dense and on the same GPU")
        ws, room = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(L.bbo_net_rms_norm_grad(dy.data_ptr(), _row(dy), pd, d_stride, h.data_ptr(), _row(h), rstd.data_ptr(), pw, rows, width, _DTYPES[dtype],
                                   dx.data_ptr(), width, pg, ws, room, _stream(stream, h)))
    return dx, dw


def quantize(x, tile=1, gate=None, want_rows=True, want_cols=False, stream=None):
    """x [rows, cols] in 8 bits: (Blocks8 of x or None, Blocks8 of its transpose or None), from one reading.

    tile: a scale for 1 x 128 values or for 128 x 128.  gate: like x; values whose gate is <= 0 count as 0 (gate = x is
    ReLU; x a gradient and gate the activation's input is ReLU's gradient)."""
    _matrix(x, "x")
    rows, cols = x.shape
    device = x.device
    pg = g_stride = 0
    if gate is not None:
        _matrix(gate, "gate", x)
        pg, g_stride = gate.data_ptr(), _row(gate)
    if tile != 1 and tile != BLOCK:
        raise ValueError("tile must be 1 or 128")
    q = empty_blocks8(rows, cols, tile, device, stream) if want_rows else None
    qt = empty_blocks8(cols, rows, tile, device, stream) if want_cols else None
    part = lambda b: (b.values.data_ptr(), _row(b.values), b.scales.data_ptr(), _row(b.scales)) if b else (0, 0, 0, 0)
    _check((_net or lib()).bbo_net_quantize(x.data_ptr(), _row(x), pg, g_stride, rows, cols, _DTYPES[x.dtype], tile, *part(q), *part(qt),
                                            _stream(stream, x)))
    return q, qt


def matmul8(a, b, dtype=torch.bfloat16, out=None, accumulate=False, workspace=None, stream=None):
    """a b^T of two Blocks8 [m, k] and [n, k] -> [m, n] in float32 or bfloat16; accumulate adds to `out`."""
    (m, k), (n, kb) = _check_blocks(a, "a"), _check_blocks(b, "b")
    av, bv = a.values, b.values
    on, device = av.get_device(), av.device
    if kb != k:
        raise ValueError("a and b must have rows of the same length")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs an output to add to")
        if dtype not in _DTYPES:
            raise ValueError("the output is float32 or bfloat16")
        out = _room(stream, (m, n), (n, 1), dtype, device)
    else:
        _matrix(out, "out")
        if out.shape != (m, n):
            raise ValueError("out must have the shape %s" % ((m, n),))
    if bv.get_device() != on or out.get_device() != on:
        raise ValueError("all tensors must be on the same GPU")
    L, ws, room = _net or lib(), 0, 0
    if workspace is None:
        need = _product_room(m, n, k)
        if need:
            workspace = _room(stream, (need,), (1,), torch.uint8, device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace must be dense and on the same GPU")
    if workspace is not None:
        ws, room = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(L.bbo_net_matmul8(av.data_ptr(), _row(av), a.scales.data_ptr(), _row(a.scales), a.tile, bv.data_ptr(), _row(bv), b.scales.data_ptr(),
                             _row(b.scales), b.tile, m, n, k, out.data_ptr(), _row(out), _DTYPES[out.dtype], accumulate, ws, room, _stream(stream, av)))
    return out


def _flat(t, name, dtypes, n=None, device=None):
    if not t.is_contiguous() or t.device.type != "cuda" or t.dtype not in dtypes or (n is not None and t.numel() != n) or \
            (device is not None and t.device != device):
        raise ValueError("%s must be dense, on the parameter's GPU, of its size and of type %s" % (name, " or ".join(map(str, dtypes))))
    return t.data_ptr()


class AdamW:
    """AdamW over a model's parameters, all tensors in a few launches.

    params: dense float32 or bfloat16 tensors (one type for all), updated in place.  lr, weight_decay: numbers, or one per
    tensor.  state: "f32" or "8bit" moments.  copies: bfloat16 copies of float32 parameters that follow them.  moments: the
    moments to start from, (m, v) or State8 per tensor; zeros by default.  step: steps already taken.  seed: of the 8-bit
    moments' rounding."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state="f32", copies=None, seed=0, moments=None,
                 step=0, stream=None):
        self.params = list(params)
        if state not in ("f32", "8bit"):
            raise ValueError("state must be f32 or 8bit")
        if len({(p.dtype, p.device) for p in self.params}) > 1:
            raise ValueError("all parameters must have one type, on one GPU")
        self.betas, self.eps, self.eight, self.seed, self.steps = betas, eps, state == "8bit", int(seed), int(step)
        n = len(self.params)
        each = lambda v: [float(x) for x in v] if isinstance(v, (list, tuple)) else [float(v)] * n
        self.lr, self.weight_decay = each(lr), each(weight_decay)
        self.copies = None if copies is None else list(copies)
        self.moments = [self._zeros(p, stream) for p in self.params] if moments is None else list(moments)
        if not len(self.lr) == len(self.weight_decay) == len(self.moments) == n or (self.copies is not None and len(self.copies) != n):
            raise ValueError("lr, weight_decay, copies and moments must have one entry per parameter")
        self._table = (Tensor * max(n, 1))()
        raw = np.frombuffer(self._table, dtype=np.uint64).reshape(-1, C.sizeof(Tensor) // 8)[:n]
        self._at, self._rates = raw[:, :2], raw[:, 8:9].view(np.float32)  # (p, g) and (lr, weight_decay) of the records
        self._sizes = [p.numel() for p in self.params]
        for i, p in enumerate(self.params):
            t, k = self._table[i], p.numel()
            t.p, t.n = _flat(p, "parameter", tuple(_DTYPES)), k
            if self.eight:
                s = self.moments[i]
                t.m, t.v = (_flat(x, "moment", (torch.float8_e4m3fn,), k, p.device) for x in (s.m, s.v))
                t.m_scales, t.v_scales = (_flat(x, "scales", (torch.float32,), -(-k // BLOCK), p.device) for x in (s.m_scales, s.v_scales))
            else:
                t.m, t.v = (_flat(x, "moment", (torch.float32,), k, p.device) for x in self.moments[i])
            if self.copies is not None:
                if p.dtype != torch.float32:
                    raise ValueError("a copy is of float32 parameters")
                t.copy = _flat(self.copies[i], "copy", (torch.bfloat16,), k, p.device)

    def _zeros(self, p, stream):
        def new(shape, dtype):
            with torch.cuda.stream(stream):
                return torch.zeros(shape, dtype=dtype, device=p.device)
        if not self.eight:
            return new(p.shape, torch.float32), new(p.shape, torch.float32)
        blocks = -(-p.numel() // BLOCK)
        codes = lambda: new(p.shape, torch.uint8).view(torch.float8_e4m3fn)
        return State8(codes(), new(blocks, torch.float32), codes(), new(blocks, torch.float32))

    def step(self, grads, grad_scale=None, stream=None):
        """One step.  grads: one dense tensor per parameter, float32 or bfloat16 (one type for all); grad_scale: float32
        [1] tensor that multiplies every gradient (clipping), or None."""
        params, n = self.params, len(self.params)
        if len(grads) != n:
            raise ValueError("one gradient per parameter")
        if not n:
            return
        dtype, device = grads[0].dtype, params[0].device
        if dtype not in _DTYPES:
            raise ValueError("gradients must be float32 or bfloat16")
        for g, size in zip(grads, self._sizes):
            if g.dtype is not dtype or g.numel() != size or not g.is_contiguous() or g.device != device:
                raise ValueError("gradients must be dense, of the parameters' sizes, of one type and on their GPU")
        self._at[:, 0] = [p.data_ptr() for p in params]
        self._at[:, 1] = [g.data_ptr() for g in grads]
        self._rates[:, 0], self._rates[:, 1] = self.lr, self.weight_decay
        scale = 0
        if grad_scale is not None:
            _vector(grad_scale.view(-1), "grad_scale", 1, params[0])
            scale = grad_scale.data_ptr()
        _check((_net or lib()).bbo_net_adamw(self._table, n, _DTYPES[params[0].dtype], _DTYPES[dtype], self.eight, self.betas[0], self.betas[1], self.eps,
                                             self.steps + 1, self.seed, scale, _stream(stream, params[0])))
        self.steps += 1
