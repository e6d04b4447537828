"""Operators beside the embedding path (include/tbe.h, last part), for models that train on histories of looked-up rows:

Scan          a gated linear recurrence over the rows of every bag, with its gradient, and its form for one new row
RelativeBias  a learned table looked up by the bucket of a distance between two rows of a history, with its gradient
AdamW         the step of a model's dense weights, many tensors in one launch, with states in 32 or 8 bits
ShortConv     a causal convolution over a few rows of every bag, with its gradient, and its form for one new row
SelectiveScan a selective state space scan over the rows of every bag, with its gradient, and its form for one new row
RMSNorm       a root-mean-square norm with the residual's addition, with its gradient, and with results in 8 bits

Argument marshalling only: every step runs in the HIP kernels of the library.  A call enqueues on the current stream, behind
this object's last call or its constructor if that was on another one (an object's calls share its scratch memory; replays of a captured graph
are the caller's to order; graphs need the objects whose calls they hold).  No call waits for the GPU, apart from `check` and a
step of `AdamW` that makes its plan anew, which no capture can hold.
What a call writes into a tensor that it was given counts for autograd as changed in place.  It may not overlap what the call reads, but for what is said to be in place.
"""
from __future__ import annotations

import ctypes as C
import math
import operator
import warnings
from typing import Dict, List, Optional, Sequence, Tuple, Union

import torch
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version as _written

from . import tbe as _tbe

DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
BLOCK = 256  # elements of a state in 8 bits that share a scale


class BiasShape(C.Structure):
    _fields_ = [("batch", C.c_int64), ("queries", C.c_int64), ("keys", C.c_int64), ("query_offset", C.c_int64),
                ("query_pos", C.c_void_p), ("key_pos", C.c_void_p), ("query_pos_stride", C.c_int64), ("key_pos_stride", C.c_int64),
                ("key_lengths", C.c_void_p), ("causal", C.c_int32), ("dtype", C.c_int32)]


class BiasStrides(C.Structure):
    _fields_ = [("sample", C.c_int64), ("head", C.c_int64), ("query", C.c_int64)]


class AdamWTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("numel", C.c_int64), ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32),
                ("weight_decay", C.c_double)]


class NormBatch(C.Structure):
    _fields_ = [("x", C.c_void_p), ("residual", C.c_void_p), ("weight", C.c_void_p), ("x_stride", C.c_int64), ("residual_stride", C.c_int64),
                ("rows", C.c_int64), ("summed", C.c_void_p), ("summed_stride", C.c_int64), ("weight_dtype", C.c_int32)]


class NormGrad(C.Structure):
    _fields_ = [("summed", C.c_void_p), ("dout", C.c_void_p), ("dsummed", C.c_void_p), ("weight", C.c_void_p), ("summed_stride", C.c_int64),
                ("dout_stride", C.c_int64), ("dsummed_stride", C.c_int64), ("rows", C.c_int64), ("rstd", C.c_void_p), ("dx", C.c_void_p),
                ("dresidual", C.c_void_p), ("dx_stride", C.c_int64), ("dresidual_stride", C.c_int64), ("dweight", C.c_void_p),
                ("weight_dtype", C.c_int32), ("residual", C.c_int32)]


class ConvBatch(C.Structure):
    _fields_ = [("x", C.c_void_p), ("x_stride", C.c_int64), ("offsets", C.c_void_p), ("bags", C.c_int64), ("rows", C.c_int64),
                ("weight", C.c_void_p), ("bias", C.c_void_p), ("before", C.c_void_p), ("weight_dtype", C.c_int32)]


class SsmBatch(C.Structure):
    _fields_ = [("x", C.c_void_p), ("delta", C.c_void_p), ("z", C.c_void_p), ("b", C.c_void_p), ("c", C.c_void_p), ("x_stride", C.c_int64),
                ("delta_stride", C.c_int64), ("z_stride", C.c_int64), ("b_stride", C.c_int64), ("c_stride", C.c_int64), ("a", C.c_void_p),
                ("skip", C.c_void_p), ("delta_bias", C.c_void_p), ("offsets", C.c_void_p), ("bags", C.c_int64), ("rows", C.c_int64),
                ("h0", C.c_void_p), ("h0_stride", C.c_int64)]


class SsmGrads(C.Structure):
    _fields_ = [("dy", C.c_void_p), ("dy_stride", C.c_int64), ("dlast", C.c_void_p), ("dx", C.c_void_p), ("ddelta", C.c_void_p),
                ("dz", C.c_void_p), ("db", C.c_void_p), ("dc", C.c_void_p), ("da", C.c_void_p), ("dskip", C.c_void_p),
                ("ddelta_bias", C.c_void_p), ("dh0", C.c_void_p)]


_ready = None  # the library object whose arguments have their types
_current_raw_stream = torch._C._cuda_getCurrentRawStream
# of a tensor, without the look for the attribute at each
_shape, _dtype, _numel = torch.Tensor.shape.__get__, torch.Tensor.dtype.__get__, torch.Tensor.numel
_address, _dense, _gpu = torch.Tensor.data_ptr, torch.Tensor.is_contiguous, torch.Tensor.get_device
_capturing = torch.cuda.is_current_stream_capturing


def _lib() -> C.CDLL:
    global _ready
    l = _tbe.lib()
    if _ready is not l:
        vp, i32, i64, f32, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_double
        batch = [vp, vp, i64, vp, i64, vp, i64, i64, vp, i64]
        l.tbe_scan_create.argtypes = [C.POINTER(vp), i32, i32, i32, i64, i64]
        l.tbe_scan_saved_floats.argtypes, l.tbe_scan_saved_floats.restype = [vp, i64], i64
        l.tbe_scan_forward.argtypes = batch + [vp, i64, vp, vp, vp]
        l.tbe_scan_backward.argtypes = batch + [vp, vp, i64, vp, vp, i64, vp, i64, vp, vp]
        l.tbe_scan_step.argtypes = [vp, vp, i64, i64, vp, vp, i64, vp, i64, i64, vp, i64, vp]
        l.tbe_bias_create.argtypes = [C.POINTER(vp), i32, C.POINTER(i64), i32, i32]
        l.tbe_bias_forward.argtypes = [vp, C.POINTER(BiasShape), vp, i32, vp, C.POINTER(BiasStrides), f32, f32, vp, C.POINTER(BiasStrides), vp]
        l.tbe_bias_backward.argtypes = [vp, C.POINTER(BiasShape), vp, C.POINTER(BiasStrides), vp, f32, vp, C.POINTER(BiasStrides), vp]
        l.tbe_adamw_create.argtypes = [C.POINTER(vp), C.POINTER(AdamWTensor), i32, i32]
        l.tbe_adamw_step.argtypes = [vp, vp, i64, f64, f64, f64, f64, C.c_uint32, vp, vp]
        l.tbe_adamw_step_counted.argtypes = [vp, vp, vp, f64, f64, f64, f64, C.c_uint32, vp, vp]
        l.tbe_scan_check.argtypes = l.tbe_conv_check.argtypes = l.tbe_ssm_check.argtypes = [vp, vp]
        l.tbe_norm_create.argtypes = [C.POINTER(vp), i32, i32, i32, f64, i64]
        l.tbe_norm_forward.argtypes = [vp, C.POINTER(NormBatch), vp, i64, vp, vp]
        l.tbe_norm_quantise.argtypes = [vp, C.POINTER(NormBatch), i32, vp, i64, vp, vp]
        l.tbe_norm_backward.argtypes = [vp, C.POINTER(NormGrad), vp]
        l.tbe_conv_create.argtypes = [C.POINTER(vp), i32, i32, i32, i32, i64, i64]
        l.tbe_conv_forward.argtypes = [vp, C.POINTER(ConvBatch), vp, i64, vp, vp]
        l.tbe_conv_backward.argtypes = [vp, C.POINTER(ConvBatch), vp, i64, vp, vp, i64, vp, vp, vp, vp]
        l.tbe_conv_step.argtypes = [vp, C.POINTER(ConvBatch), vp, i64, vp, vp, i64, vp]
        l.tbe_ssm_create.argtypes = [C.POINTER(vp), i32, i32, i32, i32, i64, i64]
        l.tbe_ssm_saved_floats.argtypes, l.tbe_ssm_saved_floats.restype = [vp, i64], i64
        l.tbe_ssm_forward.argtypes = [vp, C.POINTER(SsmBatch), vp, i64, vp, vp, vp]
        l.tbe_ssm_backward.argtypes = [vp, C.POINTER(SsmBatch), vp, C.POINTER(SsmGrads), vp]
        l.tbe_ssm_step.argtypes = [vp, C.POINTER(SsmBatch), vp, i64, i64, vp, vp, i64, vp]
        for n in ("tbe_scan_destroy", "tbe_bias_destroy", "tbe_adamw_destroy", "tbe_norm_destroy", "tbe_conv_destroy", "tbe_ssm_destroy"):
            getattr(l, n).argtypes = [vp]
        _ready = l
    return l


class _Handle:
    _destroy = ""

    def __init__(self):
        self._h = C.c_void_p()
        self.device = torch.device("cuda", torch.cuda.current_device())
        # the stream of the last call; before the first one that of the constructor, which fills states and copies there
        self._last = torch.cuda.current_stream(self.device)

    def _check(self, rc: int, what: str):
        if rc < 0:
            raise _tbe.TbeError(rc, what, _lib().tbe_last_error(None).decode())
        return rc

    def _stream(self) -> int:
        """the current stream, for the next call: behind this object's last call on another one"""
        current = _current_raw_stream(self.device.index)
        if self._last.cuda_stream != current:
            if _capturing():
                return current
            stream = torch.cuda.current_stream(self.device)
            stream.wait_stream(self._last)
            self._last = stream
        return current

    def _tensor(self, name: str, t: torch.Tensor, dtype: torch.dtype, shape) -> int:
        """address of a tensor whose type, device and shape have been looked at"""
        if t.dtype != dtype or t.device != self.device or t.shape != shape:
            raise ValueError(f"{name}: {dtype} {tuple(shape)} on {self.device} is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _whole(self, name: str, t: torch.Tensor, dtype: torch.dtype, shape) -> int:
        """the same of a tensor whose elements lie one behind another"""
        if not t.is_contiguous():
            raise ValueError(f"{name}: contiguous")
        return self._tensor(name, t, dtype, shape)

    def _rows_of(self, name: str, t: torch.Tensor, n: int, dim: int, dtype: torch.dtype) -> Tuple[int, int]:
        """address of rows of `dim` elements that lie side by side, and how far apart the rows are"""
        if _dtype(t) is not dtype or _shape(t) != (n, dim) or _gpu(t) != self.device.index:
            self._tensor(name, t, dtype, (n, dim))
        if _dense(t):
            return _address(t), dim
        if dim > 1 and n and t.stride(1) != 1:
            raise ValueError(f"{name}: the elements of a row lie side by side")
        return _address(t), (t.stride(0) if n > 1 else dim)

    def _offsets(self, offsets: torch.Tensor) -> Tuple[int, int]:
        """number of bags, address"""
        bags = offsets.numel() - 1
        if not offsets.is_contiguous() or offsets.dim() != 1 or bags < 0:
            raise ValueError("offsets: a contiguous vector of bags + 1 numbers")
        return bags, self._tensor("offsets", offsets, torch.int64, (bags + 1,))

    def _slots(self, slots: Optional[torch.Tensor], n: int) -> Optional[int]:
        return self._whole("slots", slots, torch.int64, (n,)) if slots is not None else None

    def _empty(self, *shape, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        return torch.empty(*shape, dtype=dtype, device=self.device)

    def _empty_as(self, x: torch.Tensor) -> torch.Tensor:
        """rows of x's number and type, one behind another"""
        return torch.empty_like(x) if _dense(x) else torch.empty(x.shape, dtype=x.dtype, device=self.device)

    def close(self):
        if self._h:
            getattr(_lib(), self._destroy)(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _ScanFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, x, u, offsets, h0):
        y, last, saved = plan.forward(x, u, offsets, h0, save=True)
        ctx.set_materialize_grads(False)
        ctx.plan = plan
        ctx.save_for_backward(x, u, offsets, h0, saved)
        return y, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dlast):
        x, u, offsets, h0, saved = ctx.saved_tensors
        dx, du, dh0 = ctx.plan.backward(x, u, offsets, saved, dy, dlast, h0)
        return None, dx, du, None, dh0


class Scan(_Handle):
    """h_t = f_t h_{t-1} + (1 - f_t) x_t (coupled), or + x_t, with f = sigmoid(u), over the rows of every bag.

    x, u: [rows, dim] of `dtype` (rows may lie apart); offsets: int64 [bags + 1] on the GPU; h0: fp32 [bags, dim] or None.
    Calling the object gives (y, last) with gradients to x, u and h0 (not with gradients of those: asking for them raises)."""
    _destroy = "tbe_scan_destroy"

    def __init__(self, dim: int, dtype: torch.dtype, max_bags: int, max_rows: int, coupled: bool = True):
        super().__init__()
        if dtype not in DTYPES:
            raise ValueError(f"rows are {', '.join(map(str, DTYPES))}: got {dtype}")
        self.dim, self.dtype = dim, dtype
        self._check(_lib().tbe_scan_create(C.byref(self._h), dim, DTYPES[dtype], int(coupled), max_bags, max_rows), "tbe_scan_create")

    def _rows(self, name: str, t: torch.Tensor, n: int, dtype=None) -> Tuple[int, int]:
        p = self._tensor(name, t, dtype or self.dtype, (n, self.dim))
        if self.dim > 1 and n and t.stride(1) != 1:
            raise ValueError(f"{name}: the elements of a row lie side by side")
        return p, (t.stride(0) if n > 1 else self.dim)

    def _batch(self, x, u, offsets, h0):
        n, bags = x.shape[0], offsets.numel() - 1
        if not offsets.is_contiguous() or offsets.dim() != 1 or bags < 0:
            raise ValueError("offsets: a contiguous vector of bags + 1 numbers")
        self._tensor("offsets", offsets, torch.int64, (bags + 1,))
        h = self._rows("h0", h0, bags, torch.float32) if h0 is not None else (None, 0)
        return n, bags, (self._h, *self._rows("x", x, n), *self._rows("u", u, n), offsets.data_ptr(), bags, n, *h)

    def forward(self, x, u, offsets, h0=None, y: Optional[torch.Tensor] = None, want_y: bool = True, save: bool = False):
        """(y, last, saved): h of every row (None without want_y), fp32 [bags, dim] after the last rows, what `backward` needs"""
        n, bags, args = self._batch(x, u, offsets, h0)
        given = y
        if y is None and want_y:
            y = torch.empty(n, self.dim, dtype=self.dtype, device=self.device)
        last = torch.empty(bags, self.dim, dtype=torch.float32, device=self.device)
        saved = torch.empty(self._check(_lib().tbe_scan_saved_floats(self._h, n), "tbe_scan_saved_floats"), dtype=torch.float32,
                            device=self.device) if save else None
        yp = self._rows("y", y, n) if y is not None else (None, 0)
        self._check(_lib().tbe_scan_forward(*args, *yp, last.data_ptr(), saved.data_ptr() if save else None, self._stream()),
                    "tbe_scan_forward")
        if given is not None:
            _written(given)
        return y, last, saved

    def backward(self, x, u, offsets, saved, dy=None, dlast=None, h0=None):
        """(dx, du, dh0); dh0 is None without h0"""
        n, bags, args = self._batch(x, u, offsets, h0)
        if self.dim > 1 and dy is not None and dy.stride(1) != 1 or dy is not None and n > 1 and dy.stride(0) < self.dim:
            dy = dy.contiguous()
        dlast = dlast.contiguous() if dlast is not None else None
        dx, du = (torch.empty(n, self.dim, dtype=self.dtype, device=self.device) for _ in range(2))
        dh0 = torch.empty(bags, self.dim, dtype=torch.float32, device=self.device) if h0 is not None else None
        want = self._check(_lib().tbe_scan_saved_floats(self._h, n), "tbe_scan_saved_floats")
        sp = self._whole("saved", saved, torch.float32, (want,))
        dyp = self._rows("dy", dy, n) if dy is not None else (None, 0)
        lp = self._tensor("dlast", dlast, torch.float32, (bags, self.dim)) if dlast is not None else None
        self._check(_lib().tbe_scan_backward(*args, sp, *dyp, lp, dx.data_ptr(), self.dim, du.data_ptr(), self.dim,
                                             dh0.data_ptr() if dh0 is not None else None, self._stream()), "tbe_scan_backward")
        return dx, du, dh0

    def __call__(self, x, u, offsets, h0=None):
        return _ScanFunction.apply(self, x, u, offsets, h0)

    def step(self, state, x, u, slots=None, y=None):
        """one more row for the states `slots` (int64; None: the first ones), in place; returns y = the new states in `dtype`"""
        n, count = x.shape[0], state.shape[0]
        args = (*self._rows("state", state, count, torch.float32), count,
                self._tensor("slots", slots, torch.int64, (n,)) if slots is not None else None, *self._rows("x", x, n), *self._rows("u", u, n))
        if slots is not None and not slots.is_contiguous():
            raise ValueError("slots: a contiguous vector")
        written = (state,) if y is None else (state, y)
        y = torch.empty(n, self.dim, dtype=self.dtype, device=self.device) if y is None else y
        yp = self._rows("y", y, n)
        self._check(_lib().tbe_scan_step(self._h, *args, n, *yp, self._stream()), "tbe_scan_step")
        _written(written)
        return y

    def check(self):
        """waits, and raises if a call had offsets that do not ascend from 0 to its rows, or a slot that is none of the states"""
        self._check(_lib().tbe_scan_check(self._h, self._stream()), "tbe_scan_check")


def log_thresholds(buckets: int, far: int) -> List[int]:
    """Distances at which the buckets 1, 2, ... of a side begin: one for each distance up to half of the buckets, the rest
    spread over the logarithm; the last bucket holds what is `far` or so and beyond."""
    exact = max(1, buckets // 2)
    t = list(range(1, exact + 1))
    for k in range(exact + 1, buckets):
        t.append(max(t[-1] + 1, math.ceil(exact * (far / exact) ** ((k - exact) / (buckets - exact)))))
    return t[:buckets - 1]


_WHERE = ("q_pos", "k_pos", "key_lengths"), ("q_offset", "causal")  # tensors and numbers that say where scores are


class _BiasFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, table, scores, where):
        ctx.plan, ctx.where, ctx.scale = plan, {k: where[k] for k in _WHERE[1] if k in where}, where.get("scale", 1.0)
        ctx.save_for_backward(*(where.get(k) for k in _WHERE[0]))
        ctx.table_dtype = table.dtype
        return plan.forward(table, scores=scores, **where)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        where = dict(zip(_WHERE[0], ctx.saved_tensors), **ctx.where)
        want_table, want_scores = ctx.needs_input_grad[1], ctx.needs_input_grad[2]
        got = ctx.plan.backward(dout, want_dtable=want_table, want_dscores=want_scores, scale=ctx.scale, **where)
        dtable, dscores = got if want_scores else (got, None)
        return None, dtable.to(ctx.table_dtype) if want_table else None, dscores, None


class RelativeBias(_Handle):
    """table[bucket of the distance of key and query, head], alone or added to scores [batch, heads, queries, keys].

    thresholds: distances at which the buckets 1, 2, ... begin (see `log_thresholds`).  bidirectional: keys after the query have
    buckets of their own; else they are at distance 0.  Calling the object gives the biased scores with gradients to the table
    and the scores (not with gradients of those: asking for them raises)."""
    _destroy = "tbe_bias_destroy"

    def __init__(self, heads: int, thresholds: Sequence[int], bidirectional: bool = False):
        super().__init__()
        self.heads, self.buckets = heads, (len(thresholds) + 1) * (2 if bidirectional else 1)
        self._check(_lib().tbe_bias_create(C.byref(self._h), heads, (C.c_int64 * max(1, len(thresholds)))(*thresholds), len(thresholds),
                                           int(bidirectional)), "tbe_bias_create")

    def _shape(self, shape, dtype, q_pos, k_pos, q_offset, key_lengths, causal):
        b, q, k = shape
        if dtype not in DTYPES:
            raise ValueError(f"scores are {', '.join(map(str, DTYPES))}: got {dtype}")

        def positions(name, t, n):
            if t is None:
                return None, 0
            p = self._tensor(name, t, torch.int64, (b, n))
            if n > 1 and t.stride(1) != 1:
                raise ValueError(f"{name}: the positions of a sample lie side by side")
            return p, (t.stride(0) if b > 1 else n)
        (qp, qs), (kp, ks) = positions("q_pos", q_pos, q), positions("k_pos", k_pos, k)
        if key_lengths is not None and not key_lengths.is_contiguous():
            raise ValueError("key_lengths: a contiguous vector")
        lp = self._tensor("key_lengths", key_lengths, torch.int64, (b,)) if key_lengths is not None else None
        return BiasShape(b, q, k, q_offset, qp, kp, qs, ks, lp, int(causal), DTYPES[dtype])

    def _scores(self, name, t, dtype, shape):
        b, q, k = shape
        p = self._tensor(name, t, dtype, (b, self.heads, q, k))
        if k > 1 and t.stride(3) != 1:
            raise ValueError(f"{name}: the keys of a query lie side by side")
        return p, BiasStrides(*t.stride()[:3])

    def forward(self, table, shape: Optional[Tuple[int, int, int]] = None, dtype: Optional[torch.dtype] = None, scores=None, scale: float = 1.0,
                q_pos=None, k_pos=None, q_offset: int = 0, key_lengths=None, causal: bool = False, mask_value: float = -math.inf, out=None):
        """scores * scale + bias, or the bias alone for shape = (batch, queries, keys); mask_value where masked.  causal masks keys at later
        positions than the query's: not those of the same time stamp, whatever their order (-inf in the scores stays -inf)"""
        if scores is not None:
            shape, dtype = (scores.shape[0], scores.shape[2], scores.shape[3]), scores.dtype
        dtype = dtype or table.dtype
        st = self._shape(shape, dtype, q_pos, k_pos, q_offset, key_lengths, causal)
        if table.dtype not in DTYPES or not table.is_contiguous():
            raise ValueError(f"table: contiguous, {', '.join(map(str, DTYPES))}")
        tp = self._tensor("table", table, table.dtype, (self.buckets, self.heads))
        sp, ss = self._scores("scores", scores, dtype, shape) if scores is not None else (None, None)
        given = out
        if out is None:
            out = torch.empty(shape[0], self.heads, shape[1], shape[2], dtype=dtype, device=self.device)
        op, os_ = self._scores("out", out, dtype, shape)
        if given is not None and any(n > 1 and s == 0 for n, s in zip(given.shape, given.stride())):
            raise ValueError("out: every score has a place of its own")
        self._check(_lib().tbe_bias_forward(self._h, C.byref(st), tp, DTYPES[table.dtype], sp, C.byref(ss) if ss else None, scale, mask_value, op,
                                            C.byref(os_), self._stream()), "tbe_bias_forward")
        if given is not None:
            _written(given)
        return out

    def backward(self, dout, q_pos=None, k_pos=None, q_offset: int = 0, key_lengths=None, causal: bool = False, want_dtable: bool = True,
                 want_dscores: bool = False, scale: float = 1.0):
        """gradient of the table, fp32; with want_dscores (that, gradient of the scores)"""
        if dout.dim() == 4 and dout.shape[3] > 1 and dout.stride(3) != 1:
            dout = dout.contiguous()
        shape = (dout.shape[0], dout.shape[2], dout.shape[3])
        st = self._shape(shape, dout.dtype, q_pos, k_pos, q_offset, key_lengths, causal)
        dp, ds = self._scores("dout", dout, dout.dtype, shape)
        dtable = torch.empty(self.buckets, self.heads, dtype=torch.float32, device=self.device) if want_dtable else None
        dscores = torch.empty(dout.shape, dtype=dout.dtype, device=self.device) if want_dscores else None
        ep, es = self._scores("dscores", dscores, dout.dtype, shape) if want_dscores else (None, None)
        self._check(_lib().tbe_bias_backward(self._h, C.byref(st), dp, C.byref(ds), dtable.data_ptr() if want_dtable else None, scale, ep,
                                             C.byref(es) if es else None, self._stream()), "tbe_bias_backward")
        return (dtable, dscores) if want_dscores else dtable

    def __call__(self, table, scores=None, **where):
        return _BiasFunction.apply(self, table, scores, where)


class AdamW(_Handle):
    """AdamW over a list of parameters, all in one launch (256 tensors a launch).

    state_bits 32, or 8: the moving averages in 8 bits with a scale for each 256 elements (see include/tbe.h).  master: fp32
    copies beside 16-bit parameters, True to make them from the parameters, or a list of tensors.  weight_decay: one number or one for each
    parameter.  grad_dtypes: types of the gradients, the parameters' own unless given (a step whose gradients have others makes the
    plan anew).  States of all parameters lie one behind another in `states` ("m", "v" and for 8 bits "m_scale", "v_scale"), each
    parameter's from a multiple of 256 elements on: that is what a checkpoint holds, with `step_count`.  capturable: the number of the step is counted on the
    GPU, in `states["step"]`, so that each replay of a captured step is a step of its own (without, all have the captured one's
    number; lr, betas and the gradients' places are the captured ones in both).  A step takes parameters, `master` and
    `states` as they are then: other tensors of the same sizes in their place, and parameters that have got other storage, make the
    plan anew."""
    _destroy = "tbe_adamw_destroy"

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: Union[float, Sequence[float]] = 0.01, state_bits: int = 32, master=None, seed: int = 0, step: int = 0,
                 states: Optional[Dict[str, torch.Tensor]] = None, grad_dtypes: Optional[Sequence[torch.dtype]] = None, capturable: bool = False):
        super().__init__()
        self._kept: List[C.c_void_p] = []  # handles of earlier plans
        self.params = list(params)
        self.lr, self.betas, self.eps, self.seed, self._steps, self.state_bits, self.capturable = lr, betas, eps, seed, step, state_bits, capturable
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(self.params)
        if len(decay) != len(self.params):
            raise ValueError("weight_decay: one number, or one for each parameter")
        for p in self.params:
            self._parameter(p)
        if master is True:
            master = [p.detach().float() if p.dtype != torch.float32 else None for p in self.params]
        self.master = list(master) if master else [None] * len(self.params)
        if len(self.master) != len(self.params):
            raise ValueError("master: one copy for each parameter")
        blocks = [-(-p.numel() // BLOCK) for p in self.params]
        total = sum(blocks)
        kinds = {"m": (torch.float32, total * BLOCK), "v": (torch.float32, total * BLOCK)} if state_bits == 32 else \
            {"m": (torch.uint8, total * BLOCK), "v": (torch.uint8, total * BLOCK), "m_scale": (torch.float32, total), "v_scale": (torch.float32, total)}
        self.states = states or {k: torch.zeros(n, dtype=d, device=self.device) for k, (d, n) in kinds.items()}
        if capturable:  # a step number among the given states goes before `step`
            self.states = {"step": torch.full((1,), step, dtype=torch.int64, device=self.device), **self.states}
        self._decay, self._blocks, self._kinds = decay, blocks, kinds
        self._grads = (C.c_void_p * max(1, len(self.params)))()
        self._grads_at, self._gpus = C.addressof(self._grads), [self.device.index] * len(self.params)
        self._nones = [None] * len(self.params)
        self._captured = False  # whether a step of this plan has been captured
        self._plan(list(grad_dtypes) if grad_dtypes is not None else [p.dtype for p in self.params])

    def close(self):
        super().close()
        while self._kept:
            _lib().tbe_adamw_destroy(self._kept.pop())

    @property
    def step_count(self) -> int:
        """steps so far (capturable: waits for them)"""
        if not self.capturable:
            return self._steps
        self._stream()
        return int(self.states["step"])

    @step_count.setter
    def step_count(self, n: int):
        self._steps = n
        if self.capturable:
            self._stream()
            self.states["step"].fill_(n)

    def _parameter(self, p):
        if p.dtype not in DTYPES or p.device != self.device or not p.is_contiguous():
            raise ValueError(f"parameters are contiguous, {', '.join(map(str, DTYPES))}, on {self.device}")

    def _tensors(self):
        """parameters, states and copies"""
        t, missing = [*self.params, *map(self.states.__getitem__, self._kinds)], [*map(operator.is_, self.master, self._nones)]
        return t + [w for w in self.master if w is not None] if False in missing else t, missing

    def _places(self):
        """what the plan holds of them, as it is now"""
        t, missing = self._tensors()
        return [*map(_numel, t)], [*map(_address, t)], [*map(_dtype, t)], [*map(_dense, t)], missing, len(self.params), len(self.master)

    def _plan(self, grad_dtypes):
        """a handle for the parameters, copies and states as they are now"""
        if len(self.params) != len(self._blocks) or len(self.master) != len(self._blocks):
            raise ValueError("as many parameters and copies as there were")
        if _capturing():
            raise RuntimeError("a plan is made outside of a capture: take a step with these parameters, states and types of gradients before it")
        a = {k: self._whole(k, self.states[k], d, (n,)) for k, (d, n) in self._kinds.items()}
        size, scale = 4 if self.state_bits == 32 else 1, self.state_bits == 8
        tensors, at = (AdamWTensor * max(1, len(self.params)))(), 0
        for i, (p, w, blocks) in enumerate(zip(self.params, self.master, self._blocks)):
            self._parameter(p)
            if -(-p.numel() // BLOCK) != blocks:
                raise ValueError(f"parameter {i}: {p.numel()} elements, its states have {blocks * BLOCK}")
            tensors[i] = AdamWTensor(p.data_ptr(), self._whole("master", w, torch.float32, p.shape) if w is not None else None,
                                     a["m"] + at * BLOCK * size, a["v"] + at * BLOCK * size, a["m_scale"] + 4 * at if scale else None,
                                     a["v_scale"] + 4 * at if scale else None, p.numel(), DTYPES[p.dtype], DTYPES[grad_dtypes[i]], self._decay[i])
            at += blocks
        held = sorted((t.data_ptr(), t.numel() * t.element_size()) for t in self._tensors()[0] if t.numel())
        if any(a + n > b for (a, n), (b, _) in zip(held, held[1:])):
            raise ValueError("parameters, copies and states that share memory (a weight that is tied to another one is given once)")
        h = C.c_void_p()
        self._check(_lib().tbe_adamw_create(C.byref(h), tensors, len(self.params), self.state_bits), "tbe_adamw_create")
        if self._h and self._captured:
            self._kept.append(self._h)  # graphs may hold steps of it
        elif self._h:
            _lib().tbe_adamw_destroy(self._h)
        self._h, self._captured, self._enqueue = h, False, _lib().tbe_adamw_step_counted if self.capturable else _lib().tbe_adamw_step
        self._planned, self._shapes, self._grad_dtypes = self._places(), [*map(_shape, self.params)], grad_dtypes

    def step(self, grads: Optional[Sequence[Optional[torch.Tensor]]] = None, lr: Optional[float] = None, grad_scale: Optional[torch.Tensor] = None):
        """grads: one for each parameter (None: its parameter stays as it is); without, the parameters' own `.grad`.
        grad_scale: an fp32 number on the GPU that all gradients are multiplied by"""
        grads = [p.grad for p in self.params] if grads is None else grads
        if len(grads) != len(self.params):
            raise ValueError("grads: one for each parameter")
        # Parameters, copies and states may have another storage than at the last step (moved to the host and back, loaded, assigned).
        places, ptrs, stream = self._places(), self._grads, self._stream()
        try:
            fine = [*map(_shape, grads)] == self._shapes and [*map(_dtype, grads)] == self._grad_dtypes and all(map(_dense, grads)) and \
                [*map(_gpu, grads)] == self._gpus
        except TypeError:  # a parameter without a gradient
            fine = False
        if not fine:
            for i, (g, p) in enumerate(zip(grads, self.params)):
                if g is not None and (g.shape != p.shape or g.device != self.device or not g.is_contiguous() or g.dtype not in DTYPES):
                    raise ValueError(f"gradient {i}: contiguous, of the parameter's shape {tuple(p.shape)}, on {self.device}")
            dtypes = [d if g is None else g.dtype for g, d in zip(grads, self._grad_dtypes)]
        if places != self._planned or not fine and dtypes != self._grad_dtypes:
            self._plan(self._grad_dtypes if fine else dtypes)
        ptrs[:] = [*map(_address, grads)] if fine else [None if g is None else g.data_ptr() for g in grads]
        if stream and _capturing():  # the default stream cannot be
            self._captured = True
            if not self.capturable:
                warnings.warn("the replays of this captured step all have its number (step_count): capturable=True counts them")
        gs = None
        if grad_scale is not None:
            gs = self._tensor("grad_scale", grad_scale, torch.float32, grad_scale.shape)
            if grad_scale.numel() != 1:
                raise ValueError("grad_scale: one number")
        number = self._whole("step", self.states["step"], torch.int64, (1,)) if self.capturable else self._steps + 1
        self._check(self._enqueue(self._h, self._grads_at, number, self.lr if lr is None else lr, *self.betas, self.eps, self.seed & 0xFFFFFFFF, gs,
                                  stream), "tbe_adamw_step")
        _written(self.params if fine else [p for p, g in zip(self.params, grads) if g is not None])
        self._steps += 1


def _own_rows(t: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """a gradient as autograd brings it (expanded, transposed), as rows of their own"""
    return t if t is None or t.is_contiguous() else t.contiguous()


class _NormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, x, weight, residual):
        out, summed, rstd = plan.forward(x, weight, residual)
        ctx.set_materialize_grads(False)
        ctx.plan, ctx.added, ctx.kinds = plan, residual is not None, (x.dtype, weight.dtype)
        ctx.save_for_backward(summed, rstd, weight)
        return (out, summed) if ctx.added else out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dsummed=None):
        summed, rstd, weight = ctx.saved_tensors
        if dout is None:
            dout = torch.zeros(summed.shape, dtype=ctx.kinds[0], device=summed.device)
        dx, dresidual, dweight = ctx.plan.backward(_own_rows(dout), summed, rstd, weight, _own_rows(dsummed), added=ctx.added)
        return None, dx, dweight.to(ctx.kinds[1]), dresidual


class RMSNorm(_Handle):
    """s = x + residual, in the residual's type; out = s / sqrt(mean(s s) + eps) * weight, row by row.

    x: [rows, dim] of `dtype` (rows may lie apart), as all rows here; residual: the same of `residual_dtype` (`dtype` or fp32; None: calls have no residual); weight: [dim].
    Calling the object gives (out, s), or out without a residual, with gradients to x, weight and residual (not with gradients of those: asking for them raises)."""
    _destroy = "tbe_norm_destroy"

    def __init__(self, dim: int, dtype: torch.dtype, max_rows: int, eps: float = 1e-6, residual_dtype: Optional[torch.dtype] = None):
        super().__init__()
        if dtype not in DTYPES or residual_dtype not in (None, dtype, torch.float32):
            raise ValueError(f"rows are {', '.join(map(str, DTYPES))}, the residual of their type or fp32: got {dtype}, {residual_dtype}")
        self.dim, self.dtype, self.residual_dtype = dim, dtype, residual_dtype
        self._check(_lib().tbe_norm_create(C.byref(self._h), dim, DTYPES[dtype], -1 if residual_dtype is None else DTYPES[residual_dtype], eps, max_rows),
                    "tbe_norm_create")

    def _weight(self, weight) -> Tuple[int, int]:
        if weight.dtype not in DTYPES:
            raise ValueError(f"weight: {', '.join(map(str, DTYPES))}")
        return self._whole("weight", weight, weight.dtype, (self.dim,)), DTYPES[weight.dtype]

    def _batch(self, x, weight, residual, summed):
        n = x.shape[0]
        (xp, xs), (wp, wt), (rp, rs), (sp, ss) = self._rows_of("x", x, n, self.dim, self.dtype), self._weight(weight), (None, 0), (None, 0)
        if residual is not None:
            if self.residual_dtype is None:
                raise ValueError("residual: the object was made without one (residual_dtype)")
            rp, rs = self._rows_of("residual", residual, n, self.dim, self.residual_dtype)
            summed = self._empty_as(residual) if summed is None else summed
            sp, ss = self._rows_of("summed", summed, n, self.dim, self.residual_dtype)
        elif summed is not None:
            raise ValueError("summed: there is no residual")
        else:
            summed = x
        return NormBatch(xp, rp, wp, xs, rs, n, sp, ss, wt), summed

    def forward(self, x, weight, residual=None, out=None, summed=None):
        """(out, summed, rstd): summed is the stored sum (x without a residual; `summed` may be `residual`), rstd fp32 [rows] what `backward` needs"""
        b, s = self._batch(x, weight, residual, summed)
        written = [t for t in (out, summed) if t is not None]
        out = self._empty_as(x) if out is None else out
        rstd = self._empty(b.rows)
        self._check(_lib().tbe_norm_forward(self._h, C.byref(b), *self._rows_of("out", out, b.rows, self.dim, self.dtype), rstd.data_ptr(), self._stream()),
                    "tbe_norm_forward")
        if written:
            _written(written)
        return out, s, rstd

    def quantise(self, x, weight, residual=None, group: int = 0, codes=None, summed=None):
        """(codes, scales, summed): out in 8 bits (torch.float8_e4m3fn) times a scale for each row (group 0) or each `group` elements of it,
        fp32 [rows, groups of a row]; no gradients"""
        b, s = self._batch(x, weight, residual, summed)
        written = [t for t in (codes, summed) if t is not None]
        codes = self._empty(b.rows, self.dim, dtype=torch.float8_e4m3fn) if codes is None else codes
        scales = self._empty(b.rows, -(-self.dim // group) if group > 0 else 1)
        self._check(_lib().tbe_norm_quantise(self._h, C.byref(b), group, *self._rows_of("codes", codes, b.rows, self.dim, torch.float8_e4m3fn),
                                             scales.data_ptr(), self._stream()), "tbe_norm_quantise")
        if written:
            _written(written)
        return codes, scales, s

    def backward(self, dout, summed, rstd, weight, dsummed=None, added: Optional[bool] = None):
        """(dx, dresidual, dweight): dresidual is None without a residual (added; True unless the object has none) and dx itself where they have one type;
        dweight fp32.  summed, rstd: what `forward` gave; dsummed: what comes to the stored sum from what else reads it"""
        added = self.residual_dtype is not None if added is None else added
        if added and self.residual_dtype is None:
            raise ValueError("added: the object was made without a residual (residual_dtype)")
        if dsummed is not None and not added:
            raise ValueError("dsummed: there is no residual")
        kind, n = self.residual_dtype if added else self.dtype, dout.shape[0]
        (sp, ss), (op, os_), (wp, wt) = self._rows_of("summed", summed, n, self.dim, kind), self._rows_of("dout", dout, n, self.dim, self.dtype), self._weight(weight)
        dp, ds = self._rows_of("dsummed", dsummed, n, self.dim, kind) if dsummed is not None else (None, 0)
        dx, dweight = self._empty(n, self.dim, dtype=self.dtype), self._empty(self.dim)
        apart = added and kind != self.dtype
        dresidual = self._empty(n, self.dim, dtype=kind) if apart else dx if added else None
        g = NormGrad(sp, op, dp, wp, ss, os_, ds, n, self._whole("rstd", rstd, torch.float32, (n,)), dx.data_ptr(),
                     dresidual.data_ptr() if apart else None, self.dim, self.dim, dweight.data_ptr(), wt, int(added))
        self._check(_lib().tbe_norm_backward(self._h, C.byref(g), self._stream()), "tbe_norm_backward")
        return dx, dresidual, dweight

    def __call__(self, x, weight, residual=None):
        return _NormFunction.apply(self, x, weight, residual)


class _ConvFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, x, offsets, weight, bias, before):
        ctx.set_materialize_grads(False)
        ctx.plan = plan
        ctx.save_for_backward(x, offsets, weight, bias, before)
        return plan.forward(x, offsets, weight, bias, before)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dlast):
        x, offsets, weight, bias, before = ctx.saved_tensors
        dy = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dy is None else _own_rows(dy)
        dx, dweight, dbias, dbefore = ctx.plan.backward(x, offsets, weight, dy, bias, before, _own_rows(dlast))
        return None, dx, None, dweight.to(weight.dtype), dbias.to(bias.dtype) if bias is not None else None, dbefore


class ShortConv(_Handle):
    """y_t = bias + sum over j < width of weight[:, j] e_{t+j}, or silu of that, over the rows of every bag, element by element, where e is `width` - 1
    earlier rows of the bag and behind them its rows.

    x: [rows, dim] of `dtype` (rows may lie apart); offsets: int64 [bags + 1] on the GPU; weight: [dim, width], bias: [dim] of its type or None; before:
    [bags, width - 1, dim] of `dtype` or None (zero).  Calling the object gives (y, last), last being `before` of the bags' continuation and the state of `step`,
    with gradients to x, weight, bias and before (not with gradients of those: asking for them raises)."""
    _destroy = "tbe_conv_destroy"

    def __init__(self, dim: int, width: int, dtype: torch.dtype, max_bags: int, max_rows: int, silu: bool = True):
        super().__init__()
        if dtype not in DTYPES:
            raise ValueError(f"rows are {', '.join(map(str, DTYPES))}: got {dtype}")
        self.dim, self.width, self.dtype = dim, width, dtype
        self._check(_lib().tbe_conv_create(C.byref(self._h), dim, width, DTYPES[dtype], int(silu), max_bags, max_rows), "tbe_conv_create")

    def _weights(self, weight, bias):
        if weight.dtype not in DTYPES:
            raise ValueError(f"weight: {', '.join(map(str, DTYPES))}")
        return (self._whole("weight", weight, weight.dtype, (self.dim, self.width)),
                self._whole("bias", bias, weight.dtype, (self.dim,)) if bias is not None else None)

    def _batch(self, x, offsets, weight, bias, before):
        n = x.shape[0]
        bags, op = self._offsets(offsets)
        bp = self._whole("before", before, self.dtype, (bags, self.width - 1, self.dim)) if before is not None else None
        return ConvBatch(*self._rows_of("x", x, n, self.dim, self.dtype), op, bags, n, *self._weights(weight, bias), bp, DTYPES[weight.dtype])

    def forward(self, x, offsets, weight, bias=None, before=None, y=None, want_last: bool = True):
        """(y, last); last is None without want_last"""
        b = self._batch(x, offsets, weight, bias, before)
        given = y
        y = self._empty_as(x) if y is None else y
        last = self._empty(b.bags, self.width - 1, self.dim, dtype=self.dtype) if want_last else None
        self._check(_lib().tbe_conv_forward(self._h, C.byref(b), *self._rows_of("y", y, b.rows, self.dim, self.dtype),
                                            last.data_ptr() if want_last else None, self._stream()), "tbe_conv_forward")
        if given is not None:
            _written(given)
        return y, last

    def backward(self, x, offsets, weight, dy, bias=None, before=None, dlast=None):
        """(dx, dweight, dbias, dbefore): dweight and dbias fp32; dbias and dbefore are None without bias and before"""
        b = self._batch(x, offsets, weight, bias, before)
        dx, dweight = self._empty(b.rows, self.dim, dtype=self.dtype), self._empty(self.dim, self.width)
        dbias = self._empty(self.dim) if bias is not None else None
        dbefore = self._empty(b.bags, self.width - 1, self.dim, dtype=self.dtype) if before is not None else None
        lp = self._whole("dlast", dlast, self.dtype, (b.bags, self.width - 1, self.dim)) if dlast is not None else None
        self._check(_lib().tbe_conv_backward(self._h, C.byref(b), *self._rows_of("dy", dy, b.rows, self.dim, self.dtype), lp, dx.data_ptr(), self.dim,
                                             dweight.data_ptr(), dbias.data_ptr() if dbias is not None else None,
                                             dbefore.data_ptr() if dbefore is not None else None, self._stream()), "tbe_conv_backward")
        return dx, dweight, dbias, dbefore

    def __call__(self, x, offsets, weight, bias=None, before=None):
        return _ConvFunction.apply(self, x, offsets, weight, bias, before)

    def step(self, state, x, weight, bias=None, slots=None, y=None):
        """one more row for the states `slots` ([states, width - 1, dim]; int64; None: the first ones), in place; returns y"""
        n = x.shape[0]
        b = ConvBatch(*self._rows_of("x", x, n, self.dim, self.dtype), None, 0, n, *self._weights(weight, bias), None, DTYPES[weight.dtype])
        written = (state,) if y is None else (state, y)
        y = self._empty_as(x) if y is None else y
        sp = self._whole("state", state, self.dtype, (state.shape[0], self.width - 1, self.dim))
        self._check(_lib().tbe_conv_step(self._h, C.byref(b), sp, state.shape[0], self._slots(slots, n), *self._rows_of("y", y, n, self.dim, self.dtype),
                                         self._stream()), "tbe_conv_step")
        _written(written)
        return y

    def check(self):
        """waits, and raises if a call had offsets that do not ascend from 0 to its rows, or a slot that is none of the states"""
        self._check(_lib().tbe_conv_check(self._h, self._stream()), "tbe_conv_check")


class _SsmFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, x, delta, a, b, c, offsets, skip, delta_bias, z, h0):
        y, last, saved = plan.forward(x, delta, a, b, c, offsets, skip, delta_bias, z, h0, save=True)
        ctx.set_materialize_grads(False)
        ctx.plan = plan
        ctx.save_for_backward(x, delta, a, b, c, offsets, skip, delta_bias, z, h0, saved)
        return y, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dlast):
        x, delta, a, b, c, offsets, skip, delta_bias, z, h0, saved = ctx.saved_tensors
        dy = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dy is None else _own_rows(dy)
        g = ctx.plan.backward(x, delta, a, b, c, offsets, saved, dy, _own_rows(dlast), skip, delta_bias, z, h0)
        return (None, *(g.get(k) for k in ("x", "delta", "a", "b", "c")), None, *(g.get(k) for k in ("skip", "delta_bias", "z", "h0")))


class SelectiveScan(_Handle):
    """With D = softplus(delta + delta_bias): h_t[n] = exp(D_t a[n]) h_{t-1}[n] + D_t b_t[n] x_t,  y_t = sum over n of c_t[n] h_t[n] + skip x_t, times silu(z_t),
    over the rows of every bag, for each element of a row.

    x, delta, z: [rows, dim], b, c: [rows, groups * states] of `dtype` (rows may lie apart); a: fp32 [dim, states], skip, delta_bias: fp32 [dim]; offsets: int64 [bags + 1]
    on the GPU; h0: fp32 [bags, dim, states] (bags may be expanded from one); skip, delta_bias, z, h0 may be None.  groups: each has a b and c of its own; more than
    one only with a multiple of 64 elements each.  Calling the object gives (y, last), last fp32 [bags, dim, states] being h0 of the bags' continuation and the
    state of `step`, with gradients to everything but offsets (not with gradients of those: asking for them raises)."""
    _destroy = "tbe_ssm_destroy"

    def __init__(self, dim: int, states: int, dtype: torch.dtype, max_bags: int, max_rows: int, groups: int = 1):
        super().__init__()
        if dtype not in DTYPES:
            raise ValueError(f"rows are {', '.join(map(str, DTYPES))}: got {dtype}")
        self.dim, self.states, self.groups, self.dtype = dim, states, groups, dtype
        self._check(_lib().tbe_ssm_create(C.byref(self._h), dim, states, groups, DTYPES[dtype], max_bags, max_rows), "tbe_ssm_create")

    def _batch(self, x, delta, a, b, c, skip, delta_bias, z, offsets=None, h0=None):
        n, d, k, dt = x.shape[0], self.dim, self.groups * self.states, self.dtype
        (xp, xs), (tp, ts), (bp, bs), (cp, cs) = self._rows_of("x", x, n, d, dt), self._rows_of("delta", delta, n, d, dt), self._rows_of("b", b, n, k, dt), \
            self._rows_of("c", c, n, k, dt)
        zp, zs = self._rows_of("z", z, n, d, dt) if z is not None else (None, 0)
        bags, op = self._offsets(offsets) if offsets is not None else (0, None)
        hp, hs = None, 0
        if h0 is not None:
            hp, hs = self._tensor("h0", h0, torch.float32, (bags, d, self.states)), h0.stride(0) if bags > 1 else d * self.states
            if bags and not h0[0].is_contiguous():
                raise ValueError("h0: the states of a bag lie one behind another")
        vector = lambda name, t: self._whole(name, t, torch.float32, (d,)) if t is not None else None  # noqa: E731
        return SsmBatch(xp, tp, zp, bp, cp, xs, ts, zs, bs, cs, self._whole("a", a, torch.float32, (d, self.states)), vector("skip", skip),
                        vector("delta_bias", delta_bias), op, bags, n, hp, hs)

    def forward(self, x, delta, a, b, c, offsets, skip=None, delta_bias=None, z=None, h0=None, y=None, want_last: bool = True, save: bool = False):
        """(y, last, saved): last fp32 [bags, dim, states] after the last rows (None without want_last), what `backward` needs"""
        t = self._batch(x, delta, a, b, c, skip, delta_bias, z, offsets, h0)
        given = y
        y = self._empty_as(x) if y is None else y
        last = self._empty(t.bags, self.dim, self.states) if want_last else None
        saved = self._empty(self._check(_lib().tbe_ssm_saved_floats(self._h, t.rows), "tbe_ssm_saved_floats")) if save else None
        self._check(_lib().tbe_ssm_forward(self._h, C.byref(t), *self._rows_of("y", y, t.rows, self.dim, self.dtype), last.data_ptr() if want_last else None,
                                           saved.data_ptr() if save else None, self._stream()), "tbe_ssm_forward")
        if given is not None:
            _written(given)
        return y, last, saved

    def backward(self, x, delta, a, b, c, offsets, saved, dy, dlast=None, skip=None, delta_bias=None, z=None, h0=None) -> Dict[str, torch.Tensor]:
        """gradients by the arguments' names: of x, delta, a, b, c and of those of skip, delta_bias, z, h0 that there are (a, skip, delta_bias, h0 fp32)"""
        t = self._batch(x, delta, a, b, c, skip, delta_bias, z, offsets, h0)
        n, d, dt = t.rows, self.dim, self.dtype
        sp = self._whole("saved", saved, torch.float32, (self._check(_lib().tbe_ssm_saved_floats(self._h, n), "tbe_ssm_saved_floats"),))
        dyp = self._rows_of("dy", dy, n, d, dt)
        lp = self._whole("dlast", dlast, torch.float32, (t.bags, d, self.states)) if dlast is not None else None
        g = {"x": self._empty(n, d, dtype=dt), "delta": self._empty(n, d, dtype=dt), "a": self._empty(d, self.states),
             "b": self._empty(n, self.groups * self.states, dtype=dt), "c": self._empty(n, self.groups * self.states, dtype=dt)}
        if skip is not None:
            g["skip"] = self._empty(d)
        if delta_bias is not None:
            g["delta_bias"] = self._empty(d)
        if z is not None:
            g["z"] = self._empty(n, d, dtype=dt)
        if h0 is not None:
            g["h0"] = self._empty(t.bags, d, self.states)
        at = {k: v.data_ptr() for k, v in g.items()}
        s = SsmGrads(*dyp, lp, *(at.get(k) for k in ("x", "delta", "z", "b", "c", "a", "skip", "delta_bias", "h0")))
        self._check(_lib().tbe_ssm_backward(self._h, C.byref(t), sp, C.byref(s), self._stream()), "tbe_ssm_backward")
        return g

    def __call__(self, x, delta, a, b, c, offsets, skip=None, delta_bias=None, z=None, h0=None):
        if not torch.is_grad_enabled() or not any(t is not None and t.requires_grad for t in (x, delta, a, b, c, skip, delta_bias, z, h0)):
            return self.forward(x, delta, a, b, c, offsets, skip, delta_bias, z, h0)[:2]  # nothing saved
        return _SsmFunction.apply(self, x, delta, a, b, c, offsets, skip, delta_bias, z, h0)

    def step(self, state, x, delta, a, b, c, skip=None, delta_bias=None, z=None, slots=None, y=None):
        """one more row for the states `slots` (fp32 [states of the store, dim, states], a store's states may lie apart; int64; None: the first ones), in place; returns y"""
        t = self._batch(x, delta, a, b, c, skip, delta_bias, z)
        n, count = t.rows, state.shape[0]
        sp = self._tensor("state", state, torch.float32, (count, self.dim, self.states))
        if count and not state[0].is_contiguous():
            raise ValueError("state: the states of a slot lie one behind another")
        written = (state,) if y is None else (state, y)
        y = self._empty_as(x) if y is None else y
        self._check(_lib().tbe_ssm_step(self._h, C.byref(t), sp, state.stride(0) if count > 1 else self.dim * self.states, count, self._slots(slots, n),
                                        *self._rows_of("y", y, n, self.dim, self.dtype), self._stream()), "tbe_ssm_step")
        _written(written)
        return y

    def check(self):
        """waits, and raises if a call had offsets that do not ascend from 0 to its rows, or a slot that is none of the states"""
        self._check(_lib().tbe_ssm_check(self._h, self._stream()), "tbe_ssm_check")
