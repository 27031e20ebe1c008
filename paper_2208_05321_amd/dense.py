"""ctypes binding of the operators beside the cached table (include/freqcache.h): token embedding, root-mean-square norm, clipping by the
global norm.  Marshalling only: shapes, types and strides are checked here, PyTorch supplies device memory and streams."""
from __future__ import annotations

import ctypes
from array import array
from operator import attrgetter

from .binding import FreqCacheError, load_library

_TYPE_NAMES = {"float32": 0, "bfloat16": 1, "float16": 2, "float8_e4m3fn": 3, "int8": 4, "int32": 5, "int64": 6}
_FLOATS = (0, 1, 2)
_MOST_DIM = 1 << 20              # columns of a row (the C ABI takes 32 bits of their number)
_INF = float("inf")
_dtype = attrgetter("dtype")


def _refuse(what: str):
    raise FreqCacheError(-1, what)


class DenseOps:
    """Operators on the caller's device tensors, on one stream.  Each method is one C-ABI call.

    The work runs on `stream` (the current stream of the constructor's call if not given).  A method called while another stream is current
    waits for that stream, and that stream waits for the method's work, so that tensors may come from, and go to, either.
    Rows are the last dimension of a tensor; its elements have to be neighbours, rows may be any distance apart.

    Autograd does not record these calls: results require no gradient, whatever the inputs do, and the gradients are calls of their own.  What a call
    writes into a tensor of the caller's (`out`, `h_out`, `grad`, clipping in place) it does see: a tensor that was saved for a backward pass and then
    written is an error there, as after torch's own in-place operations."""

    def __init__(self, stream=None):
        import torch

        if not torch.cuda.is_available():
            raise FreqCacheError(-8, "no GPU visible; this library has no CPU path")
        self._L = load_library()
        self._torch = torch
        self._written = torch.autograd.graph.increment_version
        self._type = {getattr(torch, name): k for name, k in _TYPE_NAMES.items()}
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.device = self.stream.device
        self._index, self._raw = self.device.index, self.stream.cuda_stream
        # the current stream as a number: a tenth of a microsecond, where torch.cuda.current_stream takes two
        self._current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            rc = self._L.dense_create(ctypes.c_void_p(self._raw), ctypes.byref(h))
        self._h = h if rc == 0 else None
        self._check(rc, "dense_create")

    def _check(self, rc: int, what: str):
        if rc != 0:
            raise FreqCacheError(rc, what)

    def close(self):
        if getattr(self, "_h", None):
            self._L.dense_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reserve(self, max_tokens: int = 0, max_rows: int = 0, max_dim: int = 0, max_tensors: int = 0):
        if not 0 <= max_dim <= _MOST_DIM or not 0 <= max_tensors < 1 << 31:
            _refuse(f"max_dim {max_dim}, max_tensors {max_tensors}")
        self._check(self._L.dense_reserve(self._h, int(max_tokens), int(max_rows), int(max_dim), int(max_tensors)), "dense_reserve")

    def check(self):
        """Waits for the stream; raises ID_OUT_OF_RANGE if a call since the last check met an id outside its table."""
        self._check(self._L.dense_check(self._h), "dense_check")

    # ---- arguments ----
    def _rows(self, t, what: str):
        """(type, rows, columns, distance of rows in elements) of a tensor whose leading dimensions have one distance between rows."""
        if t.get_device() != self._index:
            _refuse(f"{what} is on {t.device}, the handle on {self.device}")
        k = self._type.get(t.dtype)
        if k is None:
            _refuse(f"{what}: type {t.dtype}")
        shape = t.shape
        if not shape or not 0 < shape[-1] <= _MOST_DIM:
            _refuse(f"{what}: shape {tuple(shape)}")
        d = shape[-1]
        n = t.numel() // d
        if t.is_contiguous() or n == 0:
            return k, n, d, d
        stride = t.stride()
        if d > 1 and stride[-1] != 1:
            _refuse(f"{what}: the elements of a row have to be neighbours")
        step, size = None, 1            # leading dimensions, innermost first
        for length, st in zip(reversed(shape[:-1]), reversed(stride[:-1])):
            if length == 1:
                continue
            if step is None:
                step = st
            elif st != step * size:
                _refuse(f"{what}: rows have to be one distance apart")
            size *= length
        if step is None:
            step = d
        if step < d:
            _refuse(f"{what}: rows overlap")
        return k, n, d, step

    def _ids(self, ids):
        if ids.get_device() != self._index:
            _refuse(f"ids are on {ids.device}, the handle on {self.device}")
        k = self._type.get(ids.dtype)
        if k != 6 and k != 5:
            _refuse(f"ids: type {ids.dtype}")
        if not ids.is_contiguous():
            _refuse("ids have to be contiguous")
        return k

    def _vector(self, t, d: int, what: str, types):
        if t.get_device() != self._index:
            _refuse(f"{what} is on {t.device}, the handle on {self.device}")
        k = self._type.get(t.dtype)
        if k not in types:
            _refuse(f"{what}: type {t.dtype}")
        if t.numel() != d or not t.is_contiguous():
            _refuse(f"{what}: {d} contiguous elements are wanted")
        return k

    def _like(self, t, dtype=None):
        """A contiguous tensor of t's shape (torch.empty_like takes half the time of torch.empty, and keeps strides)."""
        if t.is_contiguous():
            return self._torch.empty_like(t, dtype=dtype)
        return self._torch.empty(t.shape, dtype=dtype or t.dtype, device=self.device)

    def _run(self, what: str, call, tensors, *args):
        """The call, in order with the current stream where that is another one than the handle's."""
        if self._current(self._index) == self._raw:
            rc = call(self._h, *args)
        else:
            cur = self._torch.cuda.current_stream(self.device)
            self.stream.wait_stream(cur)
            rc = call(self._h, *args)
            for t in tensors:
                for x in (t if isinstance(t, (list, tuple)) else (t,)):
                    if x is not None:
                        x.record_stream(self.stream)
            cur.wait_stream(self.stream)
        if rc != 0:
            raise FreqCacheError(rc, what)

    # ---- token embedding ----
    def token_embed_fwd(self, table, ids, scale: float = 1.0, out=None, out_dtype=None):
        """scale * table[ids]: table [rows, dim] (f32, bf16, f16), ids of any shape (int32, int64) -> ids.shape + [dim]."""
        torch = self._torch
        if table.dim() != 2:
            _refuse("table: [rows, dim] is wanted")
        tk, rows, d, ts = self._rows(table, "table")
        ik, n = self._ids(ids), ids.numel()
        given = out is not None
        if not given:
            out = torch.empty((*ids.shape, d), dtype=out_dtype or table.dtype, device=self.device)
            ok, os = self._type.get(out.dtype), d
        else:
            if out.shape != (*ids.shape, d) or (out_dtype is not None and out.dtype != out_dtype):
                _refuse("out: another shape or type")
            ok, _, _, os = self._rows(out, "out")
        if tk not in _FLOATS or ok not in _FLOATS:
            _refuse(f"types {table.dtype} -> {out.dtype}")
        self._run("token_embed_fwd", self._L.token_embed_fwd, (table, ids, out), table.data_ptr(), tk, ts, rows, d, ids.data_ptr(), ik, n, scale,
                  out.data_ptr(), ok, os)
        if given:
            self._written(out)
        return out

    def token_embed_bwd(self, grad_out, ids, num_rows: int, scale: float = 1.0, padding_id: int = -1, grad=None, grad_dtype=None,
                        accumulate: bool = False):
        """Gradient of the table [num_rows, dim]: scale * the sums of grad_out's rows by id, in f32 (default) or grad_out's type; accumulate
        adds them to `grad`, whose rows without tokens are then left alone."""
        torch = self._torch
        gk, n, d, gs = self._rows(grad_out, "grad_out")
        ik = self._ids(ids)
        if n != ids.numel() or gk not in _FLOATS:
            _refuse(f"grad_out {tuple(grad_out.shape)} {grad_out.dtype} for ids {tuple(ids.shape)}")
        given = grad is not None
        if not given:
            if accumulate:
                _refuse("accumulate needs grad")
            grad = torch.empty((num_rows, d), dtype=grad_dtype or torch.float32, device=self.device)
            tk, ts = self._type.get(grad.dtype), d
        else:
            if grad.shape != (num_rows, d) or (grad_dtype is not None and grad.dtype != grad_dtype):
                _refuse("grad: another shape or type")
            tk, _, _, ts = self._rows(grad, "grad")
        if tk != 0 and tk != gk:
            _refuse(f"types {grad_out.dtype} -> {grad.dtype}")
        self._run("token_embed_bwd", self._L.token_embed_bwd, (grad_out, ids, grad), grad_out.data_ptr(), gk, gs, ids.data_ptr(), ik, n, num_rows, d,
                  scale, padding_id, grad.data_ptr(), tk, ts, 1 if accumulate else 0)
        if given:
            self._written(grad)
        return grad

    # ---- root-mean-square norm ----
    def rms_norm_fwd(self, x, weight, residual=None, eps: float = 1e-6, out_dtype=None, group: int = 0, h_out=None, out=None):
        """(y, h, scales): h = x + residual (x itself without one), y = h * rsqrt(mean(h^2) + eps) * weight over the last dimension.
        out_dtype float8_e4m3fn or int8: y ~ q * scale with scales [..., groups] (f32) of `group` columns, or of the row (0); else scales is None.
        h_out may be x or residual."""
        torch = self._torch
        k, n, d, xs = self._rows(x, "x")
        wk = self._vector(weight, d, "weight", (0, k))
        if k not in _FLOATS:
            _refuse(f"x: type {x.dtype}")
        rs = hs = d
        h, hp, rp = x, None, None
        if residual is not None:
            rk, _, _, rs = self._rows(residual, "residual")
            if rk != k or residual.shape != x.shape:
                _refuse("residual: another shape or type than x")
            rp = residual.data_ptr()
            if h_out is None:
                h = self._like(x)
            else:
                h = h_out
                hk, _, _, hs = self._rows(h, "h_out")
                if hk != k or h.shape != x.shape:
                    _refuse("h_out: another shape or type than x")
            hp = h.data_ptr()
        elif h_out is not None:
            _refuse("h_out without residual: h is x")
        if out is None:
            y = self._like(x, out_dtype)
            yk, ys = self._type.get(y.dtype), d
        else:
            y = out
            yk, _, _, ys = self._rows(y, "out")
        if y.shape != x.shape or (out_dtype is not None and y.dtype != out_dtype) or yk not in (k, 3, 4):
            _refuse(f"out: {tuple(y.shape)} {y.dtype}")
        scales = None
        if yk >= 3:
            if group not in (0, 32, 64, 128, 256):
                _refuse(f"group {group}")
            scales = torch.empty((*x.shape[:-1], -(-d // group) if group else 1), dtype=torch.float32, device=self.device)
        elif group:
            _refuse("group without a result in 8 bits")
        self._run("rms_norm_fwd", self._L.rms_norm_fwd, (x, weight, residual, h, y, scales), x.data_ptr(), k, xs, rp, rs, weight.data_ptr(), wk, n, d, eps,
                  hp, hs, y.data_ptr(), yk, ys, scales.data_ptr() if scales is not None else None, group)
        if h_out is not None:
            self._written(h_out)
        if out is not None:
            self._written(out)
        return y, h, scales

    def rms_norm_bwd(self, grad_y, h, weight, grad_h=None, eps: float = 1e-6, grad_weight_dtype=None, out=None):
        """(grad_x, grad_weight): the gradient of x and of residual alike, and the weight's (in weight's type if not given).  grad_h: the
        gradient that arrives at h by other paths, added.  `out` (for grad_x) may be grad_y or grad_h."""
        torch = self._torch
        k, n, d, hs = self._rows(h, "h")
        yk, _, _, ys = self._rows(grad_y, "grad_y")
        wk = self._vector(weight, d, "weight", (0, k))
        if k not in _FLOATS or yk != k or grad_y.shape != h.shape:
            _refuse(f"grad_y {tuple(grad_y.shape)} {grad_y.dtype} for h {tuple(h.shape)} {h.dtype}")
        gs, gp = d, None
        if grad_h is not None:
            gk, _, _, gs = self._rows(grad_h, "grad_h")
            if gk != k or grad_h.shape != h.shape:
                _refuse("grad_h: another shape or type than h")
            gp = grad_h.data_ptr()
        if out is None:
            dx, ds = self._like(h), d
        else:
            dx = out
            dk, _, _, ds = self._rows(dx, "out")
            if dk != k or dx.shape != h.shape:
                _refuse("out: another shape or type than h")
        dw = torch.empty(d, dtype=grad_weight_dtype or weight.dtype, device=self.device)
        wt = self._type.get(dw.dtype)
        if wt not in _FLOATS:
            _refuse(f"grad_weight: type {dw.dtype}")
        self._run("rms_norm_bwd", self._L.rms_norm_bwd, (grad_y, h, weight, grad_h, dx, dw), grad_y.data_ptr(), ys, h.data_ptr(), k, hs, weight.data_ptr(),
                  wk, gp, gs, n, d, eps, dx.data_ptr(), ds, dw.data_ptr(), wt)
        if out is not None:
            self._written(out)
        return dx, dw

    # ---- clipping ----
    def _tensors(self, tensors, what: str):
        """(addresses, sizes, types) of contiguous tensors, as lists."""
        T = self._torch.Tensor                  # (one pass of C code for each question: a model has hundreds of tensors)
        kinds = list(map(self._type.get, map(_dtype, tensors)))
        if not all(map(T.is_contiguous, tensors)):
            _refuse(f"{what}: tensors have to be contiguous")
        if not {0, 1, 2}.issuperset(kinds) or not {self._index}.issuperset(map(T.get_device, tensors)):
            _refuse(f"{what}: f32, bf16 or f16 on {self.device} is wanted")
        return array("Q", map(T.data_ptr, tensors)), array("q", map(T.numel, tensors)), kinds

    def grad_norm_clip(self, grads, max_norm: float, out=None):
        """Global norm of the tensors (f32 [1]), which are scaled by min(1, max_norm / (norm + 1e-6)), in place or into the tensors of `out`."""
        torch = self._torch
        grads = list(grads)
        src, sizes, kinds = self._tensors(grads, "grads")
        dst = None
        if out is not None:
            out = list(out)
            dst, out_sizes, out_kinds = self._tensors(out, "out")
            if out_sizes != sizes or out_kinds != kinds:
                _refuse("out: other sizes or types than grads")
        if not max_norm > 0:
            _refuse(f"max_norm {max_norm}")
        kinds = array("i", kinds)
        norm = torch.empty(1, dtype=torch.float32, device=self.device)
        self._run("grad_norm_clip", self._L.grad_norm_clip, (grads, out or (), (norm,)), src.buffer_info()[0],
                  dst.buffer_info()[0] if dst is not None else None, sizes.buffer_info()[0], kinds.buffer_info()[0], len(grads), max_norm, norm.data_ptr())
        if out is not None:
            self._written(out)
        elif max_norm != _INF:
            self._written(grads)
        return norm
