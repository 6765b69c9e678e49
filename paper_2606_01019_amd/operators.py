"""Operators of an expert layer over torch tensors (include/hvd.h): routing,
the products of the chosen experts, and the norms around a block.

Each call enqueues hand-written HIP kernels on torch's current stream of its
tensors' device and returns without waiting; results are new tensors unless
``out``-style arguments are given.  Calls may be captured into a graph.  There
is no derivative: arguments that require a gradient or have a tangent are
refused.
"""

import ctypes
import operator
import struct

from .hvd import HVD_ERR_ARG, SCORES, HvdError, RouteConfig, _check, load_library


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


# Limits of include/hvd.h that are checked here too: a size that is handed over as
# 32 bits would come out as another one, within them.
MAX_ROWS, MAX_EXPERT_ROWS, MAX_EXPERTS, MAX_DIM = 1 << 23, 1 << 18, 512, 16384

# the same structure as bytes: a microsecond faster to fill than its fields
_pack_norm = struct.Struct("@PqPqPqqPPPqPqiiiiff").pack
assert len(_pack_norm(*[0] * 19)) == ctypes.sizeof(BlockNormArgs)


def _refuse(msg):
    raise HvdError(HVD_ERR_ARG, msg)


# The calls below are a few microseconds of host time each, of which a decode
# step makes dozens: torch is looked up once, configs are built once, and the
# current device and raw stream are asked for without making objects.
torch = _forward_ad = None
_codes, _configs = {}, {}


def _library():
    global torch, _forward_ad
    lib = load_library()
    if torch is None:
        import torch as t
        import torch.autograd.forward_ad as _forward_ad
        _codes.update({t.float16: 0, t.bfloat16: 1, t.float32: 2})
        torch = t
    return lib


def _dtype(t, what):
    c = _codes.get(t)
    if c is None:
        _refuse(f"{what} must be float16, bfloat16 or float32, not {t}")
    return c


def _no_grad(t, what):
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(f"{what} requires a gradient: these operators have no backward pass (use torch.no_grad())")


def _no_tangents(*args):
    """For calls inside a forward-mode level: a tangent would get lost."""
    for t in args:
        if isinstance(t, torch.Tensor) and _forward_ad.unpack_dual(t).tangent is not None:
            _refuse("an argument has a tangent: these operators have no forward-mode derivative")


def _written(t):
    """t was written in place: autograd refuses a backward pass that saved it."""
    torch.autograd.graph.increment_version(t)


def _number(v, what):
    """The float that an argument other than one stands for.  A tensor's value is
    taken now; one that requires a gradient is refused like any other."""
    if isinstance(v, torch.Tensor):
        _no_grad(v, what)
    try:
        return float(v)
    except (TypeError, ValueError, RuntimeError, OverflowError):
        _refuse(f"{what} must be a number")


def _integer(v, what):
    try:
        return operator.index(v)
    except TypeError:
        _refuse(f"{what} must be an integer")


def _matrix(t, what, device=None, rows=None, cols=None):
    """Checks a [rows, cols] tensor with unit column stride; returns its row stride."""
    if t.dim() != 2 or not t.is_cuda or (device is not None and t.device != device):
        _refuse(f"{what} must be a matrix on the GPU, on one device with the other arguments")
    if t.requires_grad:
        _no_grad(t, what)
    n, m = t.shape
    if (rows is not None and n != rows) or (cols is not None and m != cols):
        _refuse(f"{what} has shape {tuple(t.shape)}, not ({rows}, {cols})")
    rs, cs = t.stride()
    if cs != 1 and m > 1:
        _refuse(f"{what} must have unit column stride")
    return rs if n > 1 else m


def _vector(t, what, n, device):
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != n or t.device != device or not t.is_contiguous():
        _refuse(f"{what} must be a contiguous float32 vector of {n} on the arguments' device")
    if t.requires_grad:
        _no_grad(t, what)
    return t.data_ptr()


def _exact(t, what, shape, dtype, device):
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        _refuse(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the arguments' device")
    if t.requires_grad:
        _no_grad(t, what)
    return t.data_ptr()


def _call(device, fn, *args):
    """fn(*args, stream) on the device's current stream, with the device current."""
    now = torch._C._cuda_getDevice()
    if now == device.index:
        st = fn(*args, torch._C._cuda_getCurrentRawStream(now))
    else:
        with torch.cuda.device(device):
            st = fn(*args, torch._C._cuda_getCurrentRawStream(device.index))
    if st:
        _check(st)


def route(logits, top_k, *, score="softmax", bias=None, n_groups=1, top_groups=1, renorm=True, scale=1.0):
    """Choose ``top_k`` experts per row of logits [rows, n_experts] (hvd_route).

    Returns (ids int32 [rows, top_k], weights float32 [rows, top_k]): best
    first, id -1 and weight 0 where no unmasked expert is left."""
    lib = _library()
    if _forward_ad._current_level >= 0:
        _no_tangents(logits, bias, scale)
    stride = _matrix(logits, "logits")
    code = _dtype(logits.dtype, "logits")
    rows, E = logits.shape
    if rows > MAX_ROWS or E > MAX_EXPERTS:
        _refuse(f"logits may have up to {MAX_ROWS} rows of up to {MAX_EXPERTS} experts")
    dev = logits.device
    # the key holds plain numbers: equal keys are equal configs, whatever becomes
    # of the objects they came from
    if type(top_k) is not int:
        top_k = _integer(top_k, "top_k")
    if type(n_groups) is not int:
        n_groups = _integer(n_groups, "n_groups")
    if type(top_groups) is not int:
        top_groups = _integer(top_groups, "top_groups")
    if type(scale) is not float:
        scale = _number(scale, "scale")
    if renorm is not True:
        renorm = bool(renorm)
    key = (E, top_k, score, n_groups, top_groups, renorm, scale)
    cfg = _configs.get(key)
    if cfg is None:
        if score not in SCORES:
            _refuse(f"score must be one of {sorted(SCORES)}")
        if not abs(scale) <= 3.4028234663852886e38:
            _refuse("scale must be finite")
        if not 1 <= top_groups <= n_groups <= E:
            _refuse("n_groups must be in [1, n_experts], top_groups in [1, n_groups]")
        if not 1 <= top_k <= 16:
            _refuse("top_k must be in [1, 16]")
        if len(_configs) >= 256:
            _configs.clear()
        # (an address that stays: the library reads the config during the call only)
        cfg = _configs[key] = ctypes.pointer(RouteConfig(E, top_k, SCORES[score], n_groups, top_groups, renorm, scale))
    bp = _vector(bias, "bias", E, dev) if bias is not None else None
    ids = torch.empty((rows, top_k), dtype=torch.int32, device=dev)
    w = torch.empty((rows, top_k), dtype=torch.float32, device=dev)
    _call(dev, lib.hvd_route, cfg, rows, logits.data_ptr(), code, stride, bp, ids.data_ptr(), w.data_ptr())
    return ids, w


class Experts:
    """The experts of one layer (hvd_experts_*): gate and up
    [n_experts, ffn_dim, d_model], down [n_experts, d_model, ffn_dim], float16
    or bfloat16, packed once.  Weights that require a gradient are packed under
    torch.no_grad() only, and such a layer runs under it only; detached ones are
    plain data.  A graph that captured calls reads the packed weights at every
    replay: close the layer after its last one."""

    def __init__(self, gate, up, down):
        self.handle = None
        self.lib = _library()
        if gate.dim() != 3 or not gate.is_cuda:
            _refuse("gate must be [n_experts, ffn_dim, d_model] on the GPU")
        if _forward_ad._current_level >= 0:
            _no_tangents(gate, up, down)
        E, F, D = gate.shape
        if max(E, F, D) >= 1 << 31:
            _refuse("n_experts must be in [1, 512], ffn_dim and d_model at most 131072")
        self.n_experts, self.ffn_dim, self.d_model = E, F, D
        self.dtype, self.device = gate.dtype, gate.device
        if torch.cuda.is_current_stream_capturing():
            _refuse("experts are packed outside of a graph's capture (the packing is waited for)")
        for t, what, shape in ((gate, "gate", (E, F, D)), (up, "up", (E, F, D)), (down, "down", (E, D, F))):
            _exact(t, what, shape, gate.dtype, gate.device)
        cfg = ExpertsConfig(E, D, F, _dtype(gate.dtype, "weights"))
        n = self.lib.hvd_experts_bytes(ctypes.byref(cfg))
        if n == 0:
            raise HvdError(HVD_ERR_ARG, self.lib.hvd_last_error().decode())
        h = ctypes.c_void_p()
        self.buf = torch.empty(n, dtype=torch.uint8, device=self.device)
        load = lambda stream: self.lib.hvd_experts_load(ctypes.byref(cfg), gate.data_ptr(), up.data_ptr(), down.data_ptr(),
                                                        self.buf.data_ptr(), n, stream, ctypes.byref(h))
        _call(self.device, load)
        self.handle = h
        self.home = torch.cuda.current_stream(self.device)
        self.home.synchronize()  # packed: later calls may run on any stream
        self.grads = gate.requires_grad or up.requires_grad or down.requires_grad
        self.sizes = {}

    def forward(self, x, ids, weights, out=None):
        """out[t] = sum_j weights[t, j] * expert ids[t, j] of x[t]; x
        [rows, d_model] of the weights' dtype, or float32 with float16
        weights; ids int32, weights float32 [rows, top_k].  An id outside
        [0, n_experts) adds nothing."""
        if self.handle is None:
            _refuse("the experts are closed")
        if self.grads and torch.is_grad_enabled():
            _refuse("the experts were packed from weights that require a gradient: these operators have no backward pass "
                    "(use torch.no_grad(), or pack detached weights)")
        if _forward_ad._current_level >= 0:
            _no_tangents(x, ids, weights, out)
        code = _dtype(x.dtype, "x")
        dev, D = self.device, self.d_model
        xs = _matrix(x, "x", dev, None, D)
        if ids.dim() != 2:
            _refuse("ids must be [rows, top_k]")
        shape = ids.shape
        T, k = shape
        if T > MAX_EXPERT_ROWS or k > 16:
            _refuse(f"ids may have up to {MAX_EXPERT_ROWS} rows of up to 16 experts")
        if T != x.shape[0]:
            _refuse("ids must have x's rows")
        ip = _exact(ids, "ids", shape, torch.int32, dev)
        wp = _exact(weights, "weights", shape, torch.float32, dev)
        n = self.sizes.get((T, k, code))
        if n is None:
            n = self.lib.hvd_experts_workspace(self.handle, T, k, code)
            if n == 0:
                raise HvdError(HVD_ERR_ARG, self.lib.hvd_last_error().decode())
            if len(self.sizes) >= 4096:
                self.sizes.clear()
            self.sizes[(T, k, code)] = n
        xp = x.data_ptr()
        if xp % 16 or xs * x.element_size() % 16:
            x = x.clone(memory_format=torch.contiguous_format)
            xp, xs = x.data_ptr(), D
        if out is None:
            dst, ds = torch.empty((T, D), dtype=x.dtype, device=dev), D
        else:
            dst, ds = out, _matrix(out, "out", dev, T, D)
            if out.dtype != x.dtype:
                _refuse("out must have x's dtype")
        work = torch.empty(n, dtype=torch.uint8, device=dev)
        _call(dev, self.lib.hvd_experts_forward, self.handle, T, k, xp, code, xs, ip, wp, dst.data_ptr(), ds,
              work.data_ptr(), n)
        if torch._C._cuda_getCurrentRawStream(dev.index) != self.home.cuda_stream and not torch.cuda.is_current_stream_capturing():
            self.buf.record_stream(torch.cuda.current_stream(dev))  # close() may give the weights back while this call runs
        if out is not None:
            _written(out)
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
    lib = _library()
    if _forward_ad._current_level >= 0:
        _no_tangents(x, y, gain, post_gain, gate, scale, eps, x_out)
    xs, xc = _matrix(x, "x"), _dtype(x.dtype, "x")
    rows, dim = x.shape
    if rows > MAX_ROWS or dim > MAX_DIM:
        _refuse(f"x may have up to {MAX_ROWS} rows of up to {MAX_DIM} columns")
    dev = x.device
    if type(scale) is not float:
        scale = _number(scale, "scale")
    if type(eps) is not float:
        eps = _number(eps, "eps")
    yp = ys = yc = gp = gr = gs = gc = op = os_ = hp = gainp = hc = 0
    h = None
    given = x_out is not None
    if y is not None:
        yp, ys, yc = y.data_ptr(), _matrix(y, "y", dev, rows, dim), _dtype(y.dtype, "y")
        if x_out is None:
            x_out, os_ = torch.empty((rows, dim), dtype=x.dtype, device=dev), dim
        else:
            os_ = _matrix(x_out, "x_out", dev, rows, dim)
            if x_out.dtype != x.dtype:
                _refuse("x_out must have x's dtype")
        op = x_out.data_ptr()
    elif gate is not None or post_gain is not None or x_out is not None:
        _refuse("gate, post_gain and x_out belong to a y")
    if gate is not None:
        if gate.device != dev:
            _refuse("gate must be on the arguments' device")
        _no_grad(gate, "gate")
        try:
            g = gate.expand(rows, dim)
        except RuntimeError:
            _refuse(f"gate of shape {tuple(gate.shape)} does not broadcast to ({rows}, {dim})")
        gr, gs = g.stride()
        if dim == 1:
            gs = 0
        elif gs not in (0, 1):
            _refuse("gate must have unit column stride")
        gp, gc = g.data_ptr(), _dtype(gate.dtype, "gate")
    if gain is not None:
        gainp = _vector(gain, "gain", dim, dev)
        h = torch.empty((rows, dim), dtype=h_dtype or x.dtype, device=dev)
        hp, hc = h.data_ptr(), _dtype(h.dtype, "h")
    pp = _vector(post_gain, "post_gain", dim, dev) if post_gain is not None else 0
    _call(dev, lib.hvd_block_norm, _pack_norm(x.data_ptr(), xs, yp, ys, gp, gr, gs, pp, gainp, op, os_, hp, dim, xc, yc,
                                              gc, hc, scale, eps), rows, dim)
    if given:
        _written(x_out)
    return (x if y is None else x_out), h
