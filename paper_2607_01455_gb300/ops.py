"""The operators around a token table's step, on torch tensors: residual
addition with the RMS norm and its gradients, 8-bit rows and the product of
8-bit integers, softmax cross-entropy with the gradient of the logits, the
global gradient norm and clipping.

    ops = Ops()
    y, h = ops.rmsnorm(x, gain, residual=res)             # hidden states for the head
    loss, nll, dlogits = ops.softmax_loss(logits, ids)    # what Ember.step_lmhead takes
    dx, dgain = ops.rmsnorm_backward(dy, h, gain)
    norm = ops.clip_grads(grads, max_norm=1.0)            # in place
    wq, ws = ops.quantize_rows(W)                         # the trained table, served in 8 bits
    q, scales, h = ops.rmsnorm_quant(x, gain, residual=res)
    logits = ops.matmul_quant(q, scales, wq, ws)

Every computation runs in libember (include/ember.h has each operator's
definition and limits); this module checks shapes, types and devices, makes
the outputs that were not passed in, and marshals the arguments.  The common
calls take a compiled form of the same steps (csrc/ops_binding.cpp) and come
here only with arguments that it passes on: those that need a larger workspace,
that have unusual strides, or that are refused.  Matrices
are 2-D with unit stride along their rows; any row stride is accepted.  Calls
run on torch's current stream, or on `stream` (a torch stream), whose memory
their outputs and workspace then come from; a tensor that another stream
still writes has to be waited for by the caller, as with any torch call.

Autograd does not see these calls: outputs carry no history even where an input
requires a gradient, and tensors written in place keep their version.  The
gradients are what rmsnorm_backward and softmax_loss return.
"""
from array import array

import torch

from .ember import (EMBER_BF16, EMBER_ERR_DTYPE, EMBER_ERR_INVALID_ARG, EMBER_F32, EMBER_I32, EMBER_I64, EMBER_OK,
                    EmberError, _check, lib, ops_binding)

_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice

_TYPES = {torch.bfloat16: EMBER_BF16, torch.float32: EMBER_F32}
_IDS = {torch.int32: EMBER_I32, torch.int64: EMBER_I64}


class _Refused(EmberError, ValueError):
    """A call that the shapes, types or devices of its tensors rule out."""

    def __init__(self, where, why, status=EMBER_ERR_INVALID_ARG):
        super().__init__(status, f"{where}: {why}")


class Ops:
    """The operators' workspace and status block on one device, for use
    on one stream (calls on different streams share the workspace: give each
    stream its own object).  The device need not be the current one.  Before a
    graph capture, make each call once."""

    def __init__(self, device="cuda"):
        dev = torch.device(device)
        if dev.type != "cuda":
            raise _Refused("Ops", f"a CUDA device is needed, not {dev}")
        self.device = torch.device("cuda", torch.cuda.current_device() if dev.index is None else dev.index)
        self._index = self.device.index
        self._lib = lib()
        self._fast = ops_binding()
        self._status = self._workspace = None  # made by the first call that needs them, on its stream
        self._at = self._bytes = 0  # the workspace's address and size
        self._kept = []
        self._sizes = {}  # workspace bytes by operator and sizes

    # ---- arguments ----

    def _matrix(self, where, name, t, types, shape=None):
        """(address, row stride) of a 2-D tensor with unit stride along its rows."""
        size, stride = t.shape, t.stride()
        if (len(size) == 2 and stride[1] == 1 and stride[0] >= size[1] > 0 and t.get_device() == self._index
                and t.dtype in types and (shape is None or size == shape)):
            return t.data_ptr(), stride[0]
        if t.device != self.device:
            raise _Refused(where, f"{name} is on {t.device}, not on {self.device}")
        if t.dtype not in types:
            raise _Refused(where, f"{name} has type {t.dtype}", EMBER_ERR_DTYPE)
        if len(size) != 2 or (shape is not None and size != shape):
            raise _Refused(where, f"{name} has shape {tuple(size)}, not {'two dimensions' if shape is None else tuple(shape)}")
        # the stride of a single row, and that along a single column, mean nothing
        if size[1] < 1 or (stride[1] != 1 and size[1] > 1) or (stride[0] < size[1] and size[0] > 1):
            raise _Refused(where, f"{name} has shape {tuple(size)} and strides {stride}: unit stride along rows that "
                                  "do not overlap is needed")
        return t.data_ptr(), max(stride[0], size[1])

    def _vector(self, where, name, t, n, types):
        if t.get_device() != self._index:
            raise _Refused(where, f"{name} is on {t.device}, not on {self.device}")
        if t.dtype not in types:
            raise _Refused(where, f"{name} has type {t.dtype}", EMBER_ERR_DTYPE)
        if t.dim() != 1 or t.numel() != n or not t.is_contiguous():
            raise _Refused(where, f"{name} has shape {tuple(t.shape)} and strides {t.stride()}, not {n} in a row")
        return t.data_ptr()

    def _gain(self, where, gain, D):
        if gain is None:
            return None, EMBER_F32
        return self._vector(where, "gain", gain, D, _TYPES), _TYPES[gain.dtype]

    def _scratch(self, bytes_of, *sizes):
        """The workspace, of at least bytes_of(*sizes) bytes."""
        nbytes = self._sizes.get((bytes_of, sizes))
        if nbytes is None:
            if len(self._sizes) >= 4096:
                self._sizes.clear()
            nbytes = self._sizes[bytes_of, sizes] = getattr(self._lib, bytes_of)(*sizes)
        w = self._workspace
        if w is None or w.numel() < nbytes:
            # a larger one, at least twice the size; the old one stays for the
            # calls in flight and the captured graphs that use it
            size = max(nbytes, 1 << 16) if w is None else max(nbytes, 2 * w.numel())
            w = torch.empty(size, dtype=torch.uint8, device=self.device)
            self._kept.append(w)
            self._workspace = w
            self._at, self._bytes = w.data_ptr(), size
        return w

    def _status_word(self):
        if self._status is None:
            self._status = torch.zeros(4, dtype=torch.int32, device=self.device)  # EMBER_STATUS_BYTES
        return self._status.data_ptr()

    def _on(self, stream=None):
        """A context in which this object's device is the current one (libember
        launches there, and the default stream's handle means that of the
        current device) and torch allocates from the stream that the call runs on."""
        if stream is None:
            return torch.cuda.device(self.device)
        if isinstance(stream, int):
            # the handle 0 is the default stream; torch would take it for none and give a new one
            stream = (torch.cuda.ExternalStream(stream, device=self.device) if stream
                      else torch.cuda.default_stream(self.device))
        elif stream.device != self.device:
            raise _Refused("stream", f"it is on {stream.device}, not on {self.device}")
        return torch.cuda.stream(stream)

    # ---- the norm ----

    def _new(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _result(self, where, t, shape, dtype, name="out"):
        """(tensor, address, row stride) of an output: `t`, or a new one without it."""
        if t is None:
            t = torch.empty(shape, dtype=dtype, device=self.device)
            return t, t.data_ptr(), shape[1]
        return t, *self._matrix(where, name, t, (dtype,), shape)

    def rmsnorm(self, x, gain, residual=None, eps=1e-6, out=None, residual_out=None, stream=None):
        """(y, h): y = gain s / sqrt(mean s^2 + eps) over the rows of s = x +
        residual, in x's type, and h = s in the residual's type (None without
        one).  out may be x, residual_out may be residual."""
        if stream is not None:
            with self._on(stream):
                return self.rmsnorm(x, gain, residual, eps, out, residual_out)
        w = "rmsnorm"
        r = self._fast.rmsnorm(self._index, x, gain, residual, eps, out, residual_out)
        if r is not None:
            return r if r.__class__ is not int else _check(r, w)
        if _current_device() != self._index:
            with self._on():
                return self.rmsnorm(x, gain, residual, eps, out, residual_out)
        px, ldx = self._matrix(w, "x", x, _TYPES)
        shape, xt = x.shape, x.dtype
        T, D = shape
        pg, gt = self._gain(w, gain, D)
        pr, ldr, rt, ph, ldh, h = self._residual(w, residual, residual_out, shape)
        y, py, ldy = self._result(w, out, shape, xt)
        _check(self._lib.ember_rmsnorm(px, ldx, _TYPES[xt], pr, ldr, rt, pg, gt, T, D, eps, ph, ldh, py, ldy,
                                       _raw_stream(self._index)), w)
        return y, h

    def _residual(self, where, residual, residual_out, shape):
        if residual is None:
            if residual_out is not None:
                raise _Refused(where, "residual_out without a residual")
            return None, 0, EMBER_F32, None, 0, None
        pr, ldr = self._matrix(where, "residual", residual, _TYPES, shape)
        rt = residual.dtype
        h, ph, ldh = self._result(where, residual_out, shape, rt, "residual_out")
        return pr, ldr, _TYPES[rt], ph, ldh, h

    def rmsnorm_quant(self, x, gain, residual=None, eps=1e-6, residual_out=None, stream=None):
        """(q, scales, h): the norm in 8 bits, y about q * scales[:, None]."""
        if stream is not None:
            with self._on(stream):
                return self.rmsnorm_quant(x, gain, residual, eps, residual_out)
        w = "rmsnorm_quant"
        r = self._fast.rmsnorm_quant(self._index, x, gain, residual, eps, residual_out)
        if r is not None:
            return r if r.__class__ is not int else _check(r, w)
        if _current_device() != self._index:
            with self._on():
                return self.rmsnorm_quant(x, gain, residual, eps, residual_out)
        px, ldx = self._matrix(w, "x", x, _TYPES)
        T, D = x.shape
        pg, gt = self._gain(w, gain, D)
        pr, ldr, rt, ph, ldh, h = self._residual(w, residual, residual_out, x.shape)
        q, ldq, scales = self._rows8(T, D)
        _check(self._lib.ember_rmsnorm_quant(px, ldx, _TYPES[x.dtype], pr, ldr, rt, pg, gt, T, D, eps, ph, ldh,
                                             q.data_ptr(), ldq, scales.data_ptr(), _raw_stream(self._index)), w)
        return q, scales, h

    def _rows8(self, T, D):
        """New 8-bit rows, each on a 16-byte boundary, and their scales."""
        ld = (D + 15) // 16 * 16
        q = self._new((T, ld), torch.int8)
        return q if ld == D else q[:, :D], ld, self._new(T, torch.float32)

    def rmsnorm_backward(self, dy, h, gain, eps=1e-6, dres=None, out=None, stream=None):
        """(dx, dgain) of the norm at h; dres, what reaches h past the norm, is
        added to dx.  out may be dy or dres."""
        if stream is not None:
            with self._on(stream):
                return self.rmsnorm_backward(dy, h, gain, eps, dres, out)
        w = "rmsnorm_backward"
        r = self._fast.rmsnorm_backward(self._index, self._at, self._bytes, dy, h, gain, eps, dres, out)
        if r is not None:
            return r if r.__class__ is not int else _check(r, w)
        if _current_device() != self._index:
            with self._on():
                return self.rmsnorm_backward(dy, h, gain, eps, dres, out)
        ph, ldh = self._matrix(w, "h", h, _TYPES)
        shape, same = h.shape, (h.dtype,)
        T, D = shape
        py, ldy = self._matrix(w, "dy", dy, same, shape)
        pr, ldr = (None, 0) if dres is None else self._matrix(w, "dres", dres, same, shape)
        pg, gt = self._gain(w, gain, D)
        dx, pd, ldd = self._result(w, out, shape, h.dtype)
        dgain = self._new(D, torch.float32)
        ws = self._scratch("ember_rmsnorm_backward_workspace_bytes", T, D)
        _check(self._lib.ember_rmsnorm_backward(py, ldy, ph, ldh, pr, ldr, _TYPES[h.dtype], pg, gt, T, D, eps, pd, ldd,
                                                dgain.data_ptr(), ws.data_ptr(), ws.numel(), _raw_stream(self._index)), w)
        return dx, dgain

    # ---- 8 bits ----

    def quantize_rows(self, x, stream=None):
        """(q, scales) of a matrix: scales = max |x| / 127 over each row, q = x
        / scales rounded to nearest even.  Rows of q start on 16 bytes."""
        if stream is not None or _current_device() != self._index:
            with self._on(stream):
                return self.quantize_rows(x)
        w = "quantize_rows"
        px, ldx = self._matrix(w, "x", x, _TYPES)
        T, D = x.shape
        q, ldq, scales = self._rows8(T, D)
        _check(self._lib.ember_quantize_rows(px, ldx, _TYPES[x.dtype], T, D, q.data_ptr(), ldq, scales.data_ptr(),
                                             _raw_stream(self._index)), w)
        return q, scales

    def dequantize_rows(self, q, scales, dtype=torch.bfloat16, out=None, stream=None):
        """q * scales[:, None] in `dtype`."""
        if stream is not None:
            with self._on(stream):
                return self.dequantize_rows(q, scales, dtype, out)
        w = "dequantize_rows"
        r = self._fast.dequantize_rows(self._index, q, scales, _TYPES.get(dtype, -1), out)
        if r is not None:
            return r if r.__class__ is not int else _check(r, w)
        if _current_device() != self._index:
            with self._on():
                return self.dequantize_rows(q, scales, dtype, out)
        pq, ldq = self._matrix(w, "q", q, (torch.int8,))
        T, D = q.shape
        ps = self._vector(w, "scales", scales, T, (torch.float32,))
        if dtype not in _TYPES:
            raise _Refused(w, f"an output of type {dtype}", EMBER_ERR_DTYPE)
        y, py, ldy = self._result(w, out, q.shape, dtype)
        _check(self._lib.ember_dequantize_rows(pq, ldq, ps, T, D, py, ldy, _TYPES[dtype], _raw_stream(self._index)), w)
        return y

    def matmul_quant(self, xq, xs, wq, ws, dtype=torch.bfloat16, out=None, stream=None):
        """out[t][v] = xs[t] ws[v] sum_k xq[t][k] wq[v][k] in `dtype`; xq (T x
        K) and wq (V x K) int8, xs and ws fp32."""
        if stream is not None:
            with self._on(stream):
                return self.matmul_quant(xq, xs, wq, ws, dtype, out)
        w = "matmul_quant"
        r = self._fast.matmul_quant(self._index, self._at, self._bytes, self._status_word(), xq, xs, wq, ws,
                                    _TYPES.get(dtype, -1), out)
        if r is not None:
            return r if r.__class__ is not int else _check(r, w)
        if _current_device() != self._index:
            with self._on():
                return self.matmul_quant(xq, xs, wq, ws, dtype, out)
        px, ldx = self._matrix(w, "xq", xq, (torch.int8,))
        T, K = xq.shape
        pw, ldw = self._matrix(w, "wq", wq, (torch.int8,))
        V = wq.shape[0]
        if wq.shape[1] != K:
            raise _Refused(w, f"rows of {K} and of {wq.shape[1]} values")
        pxs = self._vector(w, "xs", xs, T, (torch.float32,))
        pws = self._vector(w, "ws", ws, V, (torch.float32,))
        if dtype not in _TYPES:
            raise _Refused(w, f"an output of type {dtype}", EMBER_ERR_DTYPE)
        o, po, ldo = self._result(w, out, (T, V), dtype)
        work = self._scratch("ember_matmul_quant_workspace_bytes", T, V, K)
        _check(self._lib.ember_matmul_quant(px, ldx, pxs, pw, ldw, pws, T, V, K, po, ldo, _TYPES[dtype],
                                            work.data_ptr(), work.numel(), self._status_word(),
                                            _raw_stream(self._index)), w)
        return o

    # ---- the loss ----

    def softmax_loss(self, logits, targets, weights=None, ignore_index=-100, reduction="mean", grad=True,
                     grad_dtype=None, out=None, stream=None):
        """(loss, nll, dlogits): softmax cross-entropy of T tokens over V
        entries.  nll per token, loss = sum w nll (over the counted tokens'
        number with reduction="mean"), dlogits the loss's gradient in
        grad_dtype (the logits' type by default), None with grad=False.
        out may be logits."""
        if stream is not None:
            with self._on(stream):
                return self.softmax_loss(logits, targets, weights, ignore_index, reduction, grad, grad_dtype, out)
        w = "softmax_loss"
        if reduction not in ("mean", "sum"):
            raise _Refused(w, f"reduction {reduction!r} is neither 'mean' nor 'sum'")
        dt = grad_dtype or (logits.dtype if out is None else out.dtype)
        r = self._fast.softmax_loss(self._index, self._at, self._bytes, self._status_word(), logits, targets, weights,
                                    ignore_index, reduction == "mean", _TYPES.get(dt, -2) if grad else -1, out)
        if r is not None:
            return r if r.__class__ is not int else _check(r, w)
        if _current_device() != self._index:
            with self._on():
                return self.softmax_loss(logits, targets, weights, ignore_index, reduction, grad, grad_dtype, out)
        pz, ldz = self._matrix(w, "logits", logits, _TYPES)
        T, V = logits.shape
        py = self._vector(w, "targets", targets, T, _IDS)
        pw = None if weights is None else self._vector(w, "weights", weights, T, (torch.float32,))
        if dt not in _TYPES:
            raise _Refused(w, f"a gradient of type {dt}", EMBER_ERR_DTYPE)
        d, pd, ldd = None, None, 0
        if grad:
            # rows of the gradient start where those of the logits do in a group
            # of 16 bytes, so that both take wide accesses
            ld = ldz if ldz < V + 64 else (V + 7) // 8 * 8
            if out is None:
                d = torch.empty_strided((T, V), (ld, 1), dtype=dt, device=self.device)
                pd, ldd = d.data_ptr(), ld
            else:
                d = out
                pd, ldd = self._matrix(w, "out", d, (dt,), logits.shape)
        loss = self._new((), torch.float32)
        nll = self._new(T, torch.float32)
        work = self._scratch("ember_softmax_loss_workspace_bytes", T)
        _check(self._lib.ember_softmax_loss(pz, ldz, _TYPES[logits.dtype], py, _IDS[targets.dtype], pw, ignore_index,
                                            int(reduction == "mean"), T, V, loss.data_ptr(), nll.data_ptr(), pd, ldd,
                                            _TYPES[dt], work.data_ptr(), work.numel(), self._status_word(),
                                            _raw_stream(self._index)), w)
        return loss, nll, d

    # ---- gradients ----

    def _list(self, where, tensors, out):
        """The host arrays of a call over many tensors: addresses, sizes, types."""
        n = len(tensors)
        here = [self._index] * n
        types = [_TYPES.get(t.dtype) for t in tensors]
        if [t.get_device() for t in tensors] != here or not all([t.is_contiguous() for t in tensors]):
            raise _Refused(where, f"gradients that are not contiguous tensors on {self.device}: "
                                  f"{[(tuple(t.shape), t.stride(), str(t.device)) for t in tensors][:8]}")
        if None in types:
            raise _Refused(where, f"a gradient of type {tensors[types.index(None)].dtype}", EMBER_ERR_DTYPE)
        numel = array("q", [t.numel() for t in tensors])
        ptrs = array("Q", [t.data_ptr() for t in tensors])
        if out is None:
            return ptrs, ptrs, numel, array("i", types)
        if len(out) != n:
            raise _Refused(where, f"{len(out)} outputs for {n} gradients")
        if ([o.shape for o in out] != [t.shape for t in tensors] or [_TYPES.get(o.dtype) for o in out] != types
                or [o.get_device() for o in out] != here or not all([o.is_contiguous() for o in out])):
            raise _Refused(where, f"an output of shape, type or device other than its gradient's, or not contiguous: "
                                  f"{[(tuple(o.shape), str(o.dtype), str(o.device)) for o in out][:8]}")
        outs, types = array("Q", [o.data_ptr() for o in out]), array("i", types)
        return ptrs, outs, numel, types

    def grad_norm(self, tensors, stream=None):
        """sqrt(sum of squares over all tensors), a scalar on the device."""
        if stream is not None:
            with self._on(stream):
                return self.grad_norm(tensors)
        w = "grad_norm"
        tensors = list(tensors)
        r = self._fast.grad_norm(self._index, self._at, self._bytes, tensors)
        if r is not None:
            return r if r.__class__ is not int else _check(r, w)
        if _current_device() != self._index:
            with self._on():
                return self.grad_norm(tensors)
        ptrs, _, numel, types = self._list(w, tensors, None)
        norm = self._new((), torch.float32)
        n = len(tensors)
        work = self._scratch("ember_clip_workspace_bytes", n)
        _check(self._lib.ember_grad_norm(n, ptrs.buffer_info()[0], numel.buffer_info()[0], types.buffer_info()[0],
                                         norm.data_ptr(), work.data_ptr(), work.numel(), _raw_stream(self._index)), w)
        return norm

    def clip_grads(self, tensors, max_norm, out=None, eps=1e-6, stream=None):
        """Multiplies every gradient by min(1, max_norm / (norm + eps)), in
        place or into the tensors of `out`; returns the norm before clipping,
        a scalar on the device."""
        if stream is not None:
            with self._on(stream):
                return self.clip_grads(tensors, max_norm, out, eps)
        w = "clip_grads"
        tensors = list(tensors)
        r = self._fast.clip_grads(self._index, self._at, self._bytes, tensors, max_norm, eps, out)
        if r is not None:
            return r if r.__class__ is not int else _check(r, w)
        if _current_device() != self._index:
            with self._on():
                return self.clip_grads(tensors, max_norm, out, eps)
        ptrs, outs, numel, types = self._list(w, tensors, out)
        norm = self._new((), torch.float32)
        n = len(tensors)
        work = self._scratch("ember_clip_workspace_bytes", n)
        _check(self._lib.ember_clip_grads(n, ptrs.buffer_info()[0], outs.buffer_info()[0], numel.buffer_info()[0],
                                          types.buffer_info()[0], max_norm, eps, norm.data_ptr(), work.data_ptr(),
                                          work.numel(), _raw_stream(self._index)), w)
        return norm

    def device_status(self, stream=None):
        """Synchronises; returns (and clears) the sticky status: EMBER_OK,
        EMBER_ERR_ID_OUT_OF_RANGE (a target) or EMBER_ERR_TIMEOUT."""
        if _current_device() != self._index:
            with self._on():
                return self.device_status(stream)
        at = _raw_stream(self._index) if stream is None else getattr(stream, "cuda_stream", stream)
        return self._lib.ember_status_read(self._status_word(), at)

    def set_wait_limit_ns(self, ns):
        """Limit of the bounded waits inside the kernels, for every call of this
        process from now on (0: the default, 2 s)."""
        _check(self._lib.ember_set_ops_wait_limit(int(ns)), "set_wait_limit_ns")
