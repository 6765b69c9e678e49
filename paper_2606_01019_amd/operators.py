"""Operators of an expert layer over torch tensors (include/hvd.h): routing,
the products of the chosen experts, and the norms around a block.

Each call enqueues hand-written HIP kernels on torch's current stream of its
tensors' device and returns without waiting; results are new tensors unless
``out``-style arguments are given.  Calls may be captured into a graph.
"""

import ctypes

from .hvd import HVD_ERR_ARG, HvdError, _check, load_library

_SCORES = {"softmax": 0, "sigmoid": 1}


class RouteConfig(ctypes.Structure):
    _fields_ = [("n_experts", ctypes.c_int32), ("top_k", ctypes.c_int32), ("score", ctypes.c_int32),
                ("n_groups", ctypes.c_int32), ("top_groups", ctypes.c_int32), ("renorm", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class ExpertsConfig(ctypes.Structure):
    _fields_ = [("n_experts", ctypes.c_int32), ("d_model", ctypes.c_int32), ("ffn_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class BlockNormArgs(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64), ("y", ctypes.c_void_p),
                ("y_stride", ctypes.c_int64), ("gate", ctypes.c_void_p), ("gate_row_stride", ctypes.c_int64),
                ("gate_col_stride", ctypes.c_int64), ("post_gain", ctypes.c_void_p), ("gain", ctypes.c_void_p),
                ("x_out", ctypes.c_void_p), ("x_out_stride", ctypes.c_int64), ("h", ctypes.c_void_p),
                ("h_stride", ctypes.c_int64), ("x_dtype", ctypes.c_int32), ("y_dtype", ctypes.c_int32),
                ("gate_dtype", ctypes.c_int32), ("h_dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("eps", ctypes.c_float)]


def _refuse(msg):
    raise HvdError(HVD_ERR_ARG, msg)


_codes = {}


def _dtype(t, what):
    if not _codes:
        import torch
        _codes.update({torch.float16: 0, torch.bfloat16: 1, torch.float32: 2})
    c = _codes.get(t)
    if c is None:
        _refuse(f"{what} must be float16, bfloat16 or float32, not {t}")
    return c


def _matrix(t, what, device=None, rows=None, cols=None):
    """Checks a [rows, cols] tensor with unit column stride; returns its row stride."""
    if t.dim() != 2 or not t.is_cuda or (device is not None and t.device != device):
        _refuse(f"{what} must be a matrix on the GPU, on one device with the other arguments")
    if (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        _refuse(f"{what} has shape {tuple(t.shape)}, not ({rows}, {cols})")
    if t.shape[1] > 1 and t.stride(1) != 1:
        _refuse(f"{what} must have unit column stride")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(t, what, n, device):
    import torch
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != n or t.device != device or not t.is_contiguous():
        _refuse(f"{what} must be a contiguous float32 vector of {n} on the arguments' device")
    return t.data_ptr()


def _exact(t, what, shape, dtype, device):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        _refuse(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the arguments' device")
    return t.data_ptr()


class _On:
    """Makes a device current for a call where it is not already."""

    def __init__(self, device):
        import torch
        self.cuda = torch.cuda
        self.index = device.index
        self.prev = None

    def __enter__(self):
        now = self.cuda.current_device()
        if self.index is not None and now != self.index:
            self.prev = now
            self.cuda.set_device(self.index)
        return self.cuda.current_stream()

    def __exit__(self, *exc):
        if self.prev is not None:
            self.cuda.set_device(self.prev)
        return False


def route(logits, top_k, *, score="softmax", bias=None, n_groups=1, top_groups=1, renorm=True, scale=1.0):
    """Choose ``top_k`` experts per row of logits [rows, n_experts] (hvd_route).

    Returns (ids int32 [rows, top_k], weights float32 [rows, top_k]): best
    first, id -1 and weight 0 where no unmasked expert is left."""
    import torch
    lib = load_library()
    stride = _matrix(logits, "logits")
    code = _dtype(logits.dtype, "logits")
    rows, E = logits.shape
    if score not in _SCORES:
        _refuse(f"score must be one of {sorted(_SCORES)}")
    if not 1 <= top_k <= 16:
        _refuse("top_k must be in [1, 16]")
    dev = logits.device
    bp = _vector(bias, "bias", E, dev) if bias is not None else None
    cfg = RouteConfig(E, top_k, _SCORES[score], n_groups, top_groups, 1 if renorm else 0, scale)
    with _On(dev) as s:
        ids = torch.empty((rows, top_k), dtype=torch.int32, device=dev)
        w = torch.empty((rows, top_k), dtype=torch.float32, device=dev)
        _check(lib.hvd_route(ctypes.byref(cfg), rows, logits.data_ptr(), code, stride, bp, ids.data_ptr(), w.data_ptr(),
                             s.cuda_stream))
    return ids, w


class Experts:
    """The experts of one layer (hvd_experts_*): gate and up
    [n_experts, ffn_dim, d_model], down [n_experts, d_model, ffn_dim], float16
    or bfloat16, packed once."""

    def __init__(self, gate, up, down):
        import torch
        self.lib = load_library()
        self.handle = None
        if gate.dim() != 3 or not gate.is_cuda:
            _refuse("gate must be [n_experts, ffn_dim, d_model] on the GPU")
        E, F, D = gate.shape
        self.n_experts, self.ffn_dim, self.d_model = E, F, D
        self.dtype, self.device = gate.dtype, gate.device
        for t, what, shape in ((gate, "gate", (E, F, D)), (up, "up", (E, F, D)), (down, "down", (E, D, F))):
            _exact(t, what, shape, gate.dtype, gate.device)
        cfg = ExpertsConfig(E, D, F, _dtype(gate.dtype, "weights"))
        n = self.lib.hvd_experts_bytes(ctypes.byref(cfg))
        if n == 0:
            raise HvdError(HVD_ERR_ARG, self.lib.hvd_last_error().decode())
        h = ctypes.c_void_p()
        with _On(self.device) as s:
            self.buf = torch.empty(n, dtype=torch.uint8, device=self.device)
            _check(self.lib.hvd_experts_load(ctypes.byref(cfg), gate.data_ptr(), up.data_ptr(), down.data_ptr(),
                                             self.buf.data_ptr(), n, s.cuda_stream, ctypes.byref(h)))
            s.synchronize()  # packed: later calls may run on any stream
            self.stream = s
        self.handle = h

    def forward(self, x, ids, weights, out=None):
        """out[t] = sum_j weights[t, j] * expert ids[t, j] of x[t]; x
        [rows, d_model] of the weights' dtype, or float32 with float16
        weights; ids int32, weights float32 [rows, top_k].  An id outside
        [0, n_experts) adds nothing."""
        import torch
        if self.handle is None:
            _refuse("the experts are closed")
        code = _dtype(x.dtype, "x")
        dev = self.device
        xs = _matrix(x, "x", dev, None, self.d_model)
        T = x.shape[0]
        if ids.dim() != 2:
            _refuse("ids must be [rows, top_k]")
        k = ids.shape[1]
        ip = _exact(ids, "ids", (T, k), torch.int32, dev)
        wp = _exact(weights, "weights", (T, k), torch.float32, dev)
        es = x.element_size()
        with _On(dev) as s:
            if x.data_ptr() % 16 or xs * es % 16:
                x = x.contiguous() if x.data_ptr() % 16 == 0 else x.clone(memory_format=torch.contiguous_format)
                xs = self.d_model
            dst = out
            if out is None:
                dst = torch.empty((T, self.d_model), dtype=x.dtype, device=dev)
            os_ = _matrix(dst, "out", dev, T, self.d_model)
            if dst.dtype != x.dtype:
                _refuse("out must have x's dtype")
            n = self.lib.hvd_experts_workspace(self.handle, T, k, code)
            if n == 0:
                raise HvdError(HVD_ERR_ARG, self.lib.hvd_last_error().decode())
            if s != self.stream and not torch.cuda.is_current_stream_capturing():
                self.buf.record_stream(s)  # close() may give the weights back while this call runs
            work = torch.empty(n, dtype=torch.uint8, device=dev)
            _check(self.lib.hvd_experts_forward(self.handle, T, k, x.data_ptr(), code, xs, ip, wp, dst.data_ptr(), os_,
                                                work.data_ptr(), n, s.cuda_stream))
        return dst

    __call__ = forward

    def close(self):
        """Release the handle and the packed weights."""
        if getattr(self, "handle", None):
            self.lib.hvd_experts_free(self.handle)
            self.handle = None
        self.buf = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def block_norm(x, y=None, *, gain=None, post_gain=None, gate=None, scale=1.0, eps=1e-5, h_dtype=None, x_out=None):
    """v = rms(y) * post_gain, x' = x + scale * gate * v, h = rms(x') * gain
    (hvd_block_norm); x, y [rows, dim], gate broadcastable to them.

    Returns (x', h).  Without a y, x' is x itself; without a gain, h is None.
    ``x_out`` (which may be x) receives x'; ``h_dtype`` defaults to x's."""
    import torch
    lib = load_library()
    rows, dim = x.shape if x.dim() == 2 else _refuse("x must be a matrix")
    dev = x.device
    a = BlockNormArgs()
    a.x, a.x_stride, a.x_dtype = x.data_ptr(), _matrix(x, "x"), _dtype(x.dtype, "x")
    a.scale, a.eps = scale, eps
    if y is not None:
        a.y, a.y_stride, a.y_dtype = y.data_ptr(), _matrix(y, "y", dev, rows, dim), _dtype(y.dtype, "y")
    elif gate is not None or post_gain is not None or x_out is not None:
        _refuse("gate, post_gain and x_out belong to a y")
    if gate is not None:
        if gate.device != dev:
            _refuse("gate must be on the arguments' device")
        try:
            g = gate.expand(rows, dim)
        except RuntimeError:
            _refuse(f"gate of shape {tuple(gate.shape)} does not broadcast to ({rows}, {dim})")
        if dim > 1 and g.stride(1) not in (0, 1):
            _refuse("gate must have unit column stride")
        a.gate, a.gate_dtype = g.data_ptr(), _dtype(gate.dtype, "gate")
        a.gate_row_stride, a.gate_col_stride = g.stride(0), g.stride(1) if dim > 1 else 0
    if post_gain is not None:
        a.post_gain = _vector(post_gain, "post_gain", dim, dev)
    h = None
    with _On(dev) as s:
        if y is not None:
            if x_out is None:
                x_out = torch.empty((rows, dim), dtype=x.dtype, device=dev)
            elif x_out.dtype != x.dtype:
                _refuse("x_out must have x's dtype")
            a.x_out, a.x_out_stride = x_out.data_ptr(), _matrix(x_out, "x_out", dev, rows, dim)
        if gain is not None:
            a.gain = _vector(gain, "gain", dim, dev)
            h = torch.empty((rows, dim), dtype=h_dtype or x.dtype, device=dev)
            a.h, a.h_stride, a.h_dtype = h.data_ptr(), dim, _dtype(h.dtype, "h")
        _check(lib.hvd_block_norm(ctypes.byref(a), rows, dim, s.cuda_stream))
    return (x if y is None else x_out), h
