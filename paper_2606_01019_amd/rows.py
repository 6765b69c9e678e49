"""Operators on the rows of several sequences over torch tensors (include/hvd.h):
keys and values into a paged cache, the attention over it, and penalties and
masks on logits -- what a verify step of a decoder that is not loaded here
needs around its matrix products.

The conventions are those of the expert layer's operators (operators.py): each
call enqueues hand-written HIP kernels on torch's current stream of its
tensors' device and returns without waiting, may be captured into a graph, and
has no derivative.  A captured call reads the batch's tensors again at every
replay.
"""

import ctypes
import struct

from . import operators as _op
from .hvd import HVD_ERR_ARG, HvdError
from .operators import _call, _dtype, _library, _no_grad, _no_tangents, _number, _refuse, _written

MAX_SEQS, MAX_STEP_ROWS, MAX_ADJUST_ROWS = 4096, 1 << 20, 1 << 16
MAX_HISTORY, MAX_BIAS, MAX_VOCAB = 983039, 2046, 1 << 24


class RowBatchC(ctypes.Structure):
    _fields_ = [("starts", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("pages", ctypes.c_void_p),
                ("tree", ctypes.c_void_p), ("pages_stride", ctypes.c_int64), ("n_seqs", ctypes.c_int32),
                ("max_pages", ctypes.c_int32)]


class PagedKVC(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("k_page_stride", ctypes.c_int64), ("k_head_stride", ctypes.c_int64),
                ("k_token_stride", ctypes.c_int64), ("v", ctypes.c_void_p), ("v_page_stride", ctypes.c_int64),
                ("v_head_stride", ctypes.c_int64), ("v_token_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class AppendArgs(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("k_row_stride", ctypes.c_int64), ("k_head_stride", ctypes.c_int64),
                ("v", ctypes.c_void_p), ("v_row_stride", ctypes.c_int64), ("v_head_stride", ctypes.c_int64),
                ("q", ctypes.c_void_p), ("q_row_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("q_out", ctypes.c_void_p), ("freqs", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("q_heads", ctypes.c_int32), ("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class AttendArgs(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("q_row_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("out_row_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64),
                ("slopes", ctypes.c_void_p), ("first", ctypes.c_void_p), ("prefix", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("cap", ctypes.c_float), ("q_heads", ctypes.c_int32),
                ("window", ctypes.c_int32)]


class AdjustArgs(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("logits_stride", ctypes.c_int64), ("out", ctypes.c_void_p),
                ("out_stride", ctypes.c_int64), ("best", ctypes.c_void_p), ("tokens", ctypes.c_void_p),
                ("history", ctypes.c_void_p), ("history_stride", ctypes.c_int64), ("history_lengths", ctypes.c_void_p),
                ("prompt_lengths", ctypes.c_void_p), ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
                ("presence", ctypes.c_void_p), ("bias_ids", ctypes.c_void_p), ("bias_ids_stride", ctypes.c_int64),
                ("bias", ctypes.c_void_p), ("bias_stride", ctypes.c_int64), ("allowed", ctypes.c_void_p),
                ("allowed_stride", ctypes.c_int64), ("vocab", ctypes.c_int32), ("max_history", ctypes.c_int32),
                ("n_bias", ctypes.c_int32), ("dtype", ctypes.c_int32)]


# the same structures as bytes: faster to fill than their fields
_pack_kv = struct.Struct("@PqqqPqqqiiiiii").pack
_pack_append = struct.Struct("@PqqPqqPqqPPPiiii").pack
_pack_attend = struct.Struct("@PqqPqqPPPffii").pack
_pack_adjust = struct.Struct("@PqPqPPPqPPPPPPqPqPqiiii").pack
assert len(_pack_kv(*[0] * 14)) == ctypes.sizeof(PagedKVC)
assert len(_pack_append(*[0] * 16)) == ctypes.sizeof(AppendArgs)
assert len(_pack_attend(*[0] * 13)) == ctypes.sizeof(AttendArgs)
assert len(_pack_adjust(*[0] * 23)) == ctypes.sizeof(AdjustArgs)


def _array(t, what, dtype, shape, device):
    """The address of a contiguous tensor of that type and shape (None: any size)."""
    if t.dtype != dtype or t.device != device or t.dim() != len(shape) or not t.is_contiguous():
        _refuse(f"{what} must be a contiguous {dtype} tensor of {len(shape)} dimension(s) on the arguments' device")
    if t.shape != shape:  # (None: any)
        for n, m in zip(t.shape, shape):
            if m is not None and n != m:
                _refuse(f"{what} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.requires_grad:
        _no_grad(t, what)
    return t.data_ptr()


def _table(t, what, dtype, rows, device):
    """Address, row stride and width of a matrix with unit column stride."""
    if t.dtype != dtype or t.device != device or t.dim() != 2 or t.shape[0] != rows:
        _refuse(f"{what} must be a {dtype} matrix of {rows} row(s) on the arguments' device")
    if t.requires_grad:
        _no_grad(t, what)
    n, m = t.shape
    rs, cs = t.stride()
    if cs != 1 and m > 1:
        _refuse(f"{what} must have unit column stride")
    return t.data_ptr(), (rs if n > 1 else m), m


def _heads(t, what, device, rows, heads, dim):
    """Row and head stride of a [rows, heads, dim] tensor."""
    if t.dim() != 3 or t.device != device:
        _refuse(f"{what} must be [rows, heads, head_dim] on the arguments' device")
    if t.requires_grad:
        _no_grad(t, what)
    n, h, d = t.shape
    if n != rows or (heads is not None and h != heads) or d != dim:
        _refuse(f"{what} has shape {tuple(t.shape)}, not ({rows}, {heads if heads is not None else 'heads'}, {dim})")
    rs, hs, cs = t.stride()
    if cs != 1 and d > 1:
        _refuse(f"{what} must have unit stride within a head")
    return rs, hs


class RowBatch:
    """The rows of one step (hvd_row_batch): sequence s has rows starts[s] ..
    starts[s + 1] - 1, and its ``lengths[s]`` keys, this step's included, lie on
    the pages ``pages[s]`` of a cache.  ``tree`` (int64, a row each): bit j says
    that row j of the sequence lies on the row's path, its own bit included.

    starts int32 [n_seqs + 1], lengths int32 [n_seqs], pages int32 [n_seqs,
    max_pages]; ``adjust_logits`` needs neither lengths nor pages.  The tensors
    are kept, not copied: calls read what they hold when they run, so one batch
    serves every layer of a step, and a captured graph the steps after it."""

    def __init__(self, starts, lengths=None, pages=None, *, tree=None):
        _library()
        torch = _op.torch
        if _op._forward_ad._current_level >= 0:
            _no_tangents(starts, lengths, pages, tree)
        if not isinstance(starts, torch.Tensor) or not starts.is_cuda or starts.dim() != 1 or starts.shape[0] < 1:
            _refuse("starts must be an int32 vector of n_seqs + 1 on the GPU")
        dev, S = starts.device, starts.shape[0] - 1
        if S > MAX_SEQS:
            _refuse(f"a batch may have up to {MAX_SEQS} sequences")
        sp = _array(starts, "starts", torch.int32, (S + 1,), dev)
        if (lengths is None) != (pages is None):
            _refuse("lengths and pages go together")
        lp = pp = ps = P = 0
        if lengths is not None:
            lp = _array(lengths, "lengths", torch.int32, (S,), dev)
            pp, ps, P = _table(pages, "pages", torch.int32, S, dev)
            if P > 1 << 25:
                _refuse("a sequence may have up to 2^25 pages")
        tp = 0
        if tree is not None:
            tp = _array(tree, "tree", torch.int64, (None,), dev)
        self.starts, self.lengths, self.pages, self.tree = starts, lengths, pages, tree
        self.device, self.n_seqs = dev, S
        self._c = RowBatchC(sp, lp, pp, tp, ps, S, P)
        self._p = ctypes.addressof(self._c)
        self._tree_rows = None if tree is None else tree.shape[0]
        self._sizes = {}

    def _check_rows(self, rows, most, keys):
        if rows > most:
            _refuse(f"a call takes up to {most} rows")
        if self._tree_rows is not None and rows != self._tree_rows:
            _refuse(f"the batch's tree has {self._tree_rows} rows, not {rows}")
        if keys and self.lengths is None:
            _refuse("the batch has no lengths and pages")


def _batch(batch):
    if not isinstance(batch, RowBatch):
        _refuse("batch must be a RowBatch")
    return batch.device


def _cache(k_cache, v_cache, dev):
    """The cache's structure, its code, heads and head dimension."""
    shape = k_cache.shape
    if k_cache.dim() != 4 or v_cache.shape != shape or k_cache.device != dev or v_cache.device != dev:
        _refuse("k_cache and v_cache must be [n_pages, n_heads, page_size, head_dim] on the batch's device")
    if v_cache.dtype != k_cache.dtype:
        _refuse("k_cache and v_cache must have one dtype")
    if k_cache.requires_grad or v_cache.requires_grad:
        _no_grad(k_cache, "k_cache")
        _no_grad(v_cache, "v_cache")
    n, h, p, d = shape
    if n >= 1 << 31 or h > 256 or p > 1024 or d > 256:
        _refuse("a cache has up to 2^31 - 1 pages of up to 1024 tokens, up to 256 heads of up to 256")
    ks, vs = k_cache.stride(), v_cache.stride()
    if (ks[3] != 1 or vs[3] != 1) and d > 1:
        _refuse("the caches must have unit stride within a head")
    code = _dtype(k_cache.dtype, "the caches")
    return _pack_kv(k_cache.data_ptr(), ks[0], ks[1], ks[2], v_cache.data_ptr(), vs[0], vs[1], vs[2], n, h, p, d, code, 0), code, h, d


def append_kv(k_cache, v_cache, k, v, batch, *, q=None, freqs=None, interleaved=False, positions=None):
    """Write the rows' keys and values [rows, n_heads, head_dim] to their places in
    the caches [n_pages, n_heads, page_size, head_dim], keys rotated on the way
    (hvd_append_kv); returns the rotated queries of ``q`` [rows, q_heads,
    head_dim] in the caches' dtype, or None.

    ``freqs`` (float64, radians per position) rotates the first 2 * len(freqs)
    columns of each head, in halves or in neighbouring pairs (``interleaved``);
    without it nothing is rotated.  ``positions`` (int32, a row each) takes the
    place of the batch's.  k, v and q have one dtype (float16, bfloat16 or
    float32) and any row and head strides; the caches share no memory."""
    _library()
    torch = _op.torch
    if _op._forward_ad._current_level >= 0:
        _no_tangents(k_cache, v_cache, k, v, q, freqs, positions)
    dev = _batch(batch)
    kv, _, H, D = _cache(k_cache, v_cache, dev)
    if k.dim() != 3:
        _refuse("k must be [rows, n_heads, head_dim]")
    rows = k.shape[0]
    batch._check_rows(rows, MAX_STEP_ROWS, True)
    kr, kh = _heads(k, "k", dev, rows, H, D)
    vr, vh = _heads(v, "v", dev, rows, H, D)
    code = _dtype(k.dtype, "k")
    if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        _refuse("k, v and q must have one dtype")
    qp = qr = qh = op = fp = pp = Hq = rot = 0
    out = None
    if q is not None:
        qr, qh = _heads(q, "q", dev, rows, None, D)
        Hq = q.shape[1]
        if not 1 <= Hq <= 256:
            _refuse("q must have from 1 to 256 heads")
        out = torch.empty((rows, Hq, D), dtype=k_cache.dtype, device=dev)
        qp, op = q.data_ptr(), out.data_ptr()
    if freqs is not None:
        fp, rot = _array(freqs, "freqs", torch.float64, (None,), dev), 2 * freqs.shape[0]
        if rot > D:
            _refuse("freqs may have up to head_dim / 2 frequencies")
    if positions is not None:
        pp = _array(positions, "positions", torch.int32, (rows,), dev)
    args = _pack_append(k.data_ptr(), kr, kh, v.data_ptr(), vr, vh, qp, qr, qh, op, fp, pp, Hq, rot, 1 if interleaved else 0, code)
    _call(dev, _library().hvd_append_kv, batch._p, kv, args, rows)
    _written(k_cache)
    _written(v_cache)
    return out


def attend(q, k_cache, v_cache, batch, *, scale=None, cap=0.0, window=0, slopes=None, first=None, prefix=None, out=None):
    """Attention of the rows' queries [rows, q_heads, head_dim] over the caches
    [n_pages, n_heads, page_size, head_dim] of the same dtype, in which their own
    keys lie already (hvd_attend); returns [rows, q_heads, head_dim].

    Scores are ``scale`` (head_dim ** -0.5) * q.k, then ``cap`` * tanh(s / cap) with a
    cap, minus ``slopes``[head] (float32) * distance.  A row sees the keys up to
    its own -- with the batch's tree, of this step's those on its path -- within
    ``window`` positions, from key ``first``[row] (int32) on, and its sequence's
    first ``prefix``[seq] (int32) keys even where they come after it.  Rows that
    see nothing, and rows of no sequence, are 0.  ``out`` (q itself, or memory
    apart from q's) receives the result."""
    lib = _library()
    torch = _op.torch
    if _op._forward_ad._current_level >= 0:
        _no_tangents(q, k_cache, v_cache, scale, cap, slopes, first, prefix, out)
    dev = _batch(batch)
    kv, code, H, D = _cache(k_cache, v_cache, dev)
    if q.dim() != 3:
        _refuse("q must be [rows, q_heads, head_dim]")
    rows, Hq = q.shape[:2]
    batch._check_rows(rows, MAX_STEP_ROWS, True)
    qr, qh = _heads(q, "q", dev, rows, None, D)
    if q.dtype != k_cache.dtype:
        _refuse("q must have the caches' dtype")
    if Hq > 256:
        _refuse("q may have up to 256 heads")
    if type(cap) is not float:
        cap = _number(cap, "cap")
    scale = D ** -0.5 if scale is None else scale if type(scale) is float else _number(scale, "scale")
    if not (abs(scale) <= 1.7014118346046923e38 and abs(cap) <= 3.4028234663852886e38):
        _refuse("scale must be in [-2^127, 2^127] and cap finite")
    if cap != 0.0 and cap < 2.0 ** -149:  # (one that is 0 in 32 bits would be none)
        _refuse("cap must be 0 or at least 2^-149")
    if type(window) is not int:
        window = _op._integer(window, "window")
    if not 0 <= window < 1 << 31:
        _refuse("window must be in [0, 2^31)")
    sp = _array(slopes, "slopes", torch.float32, (Hq,), dev) if slopes is not None else 0
    fp = _array(first, "first", torch.int32, (rows,), dev) if first is not None else 0
    pp = _array(prefix, "prefix", torch.int32, (batch.n_seqs,), dev) if prefix is not None else 0
    key = (rows, Hq, H, D, k_cache.shape[2])
    n = batch._sizes.get(key)
    if n is None:
        n = lib.hvd_attend_workspace(batch._p, kv, Hq, rows)
        if n == 0:
            raise HvdError(HVD_ERR_ARG, lib.hvd_last_error().decode())
        if len(batch._sizes) >= 256:
            batch._sizes.clear()
        batch._sizes[key] = n
    qp = q.data_ptr()
    dst = out
    if out is None:
        dst = torch.empty((rows, Hq, D), dtype=q.dtype, device=dev)
        outr, outh = Hq * D, D
    else:
        outr, outh = _heads(out, "out", dev, rows, Hq, D)
        if out.dtype != q.dtype:
            _refuse("out must have q's dtype")
    if qp % 16 or qr % 8 or qh % 8:
        q = q.clone(memory_format=torch.contiguous_format)
        qp, qr, qh = q.data_ptr(), Hq * D, D
    work = torch.empty(n, dtype=torch.uint8, device=dev) if n > 16 else None
    args = _pack_attend(qp, qr, qh, dst.data_ptr(), outr, outh, sp, fp, pp, scale, cap, Hq, window)
    _call(dev, lib.hvd_attend, batch._p, kv, args, rows, 0 if work is None else work.data_ptr(), n)
    if out is not None:
        _written(out)
    return dst


def _per_seq(v, what, n, dev):
    return 0 if v is None else _array(v, what, _op.torch.float32, (n,), dev)


def adjust_logits(logits, batch, *, tokens=None, history=None, history_lengths=None, prompt_lengths=None, repetition=None,
                  frequency=None, presence=None, bias_ids=None, bias=None, allowed=None, out=None, write=True):
    """Penalties, biases and a mask on the rows' logits [rows, vocab], and each
    row's best token (hvd_adjust_logits); returns (adjusted logits or None, best
    int32 [rows]).

    A token counts as seen if it lies in its sequence's ``history`` (int32
    [n_seqs, n], the first ``history_lengths``[seq] of them) or in ``tokens``
    (int32, this step's row each) on the row's own path; as generated unless it
    lies only in the first ``prompt_lengths``[seq] of the history.  Per sequence
    (float32): ``repetition`` divides positive and multiplies other logits of seen
    tokens, ``frequency`` is taken off once for each time a token was generated,
    ``presence`` if it was at all.  ``bias`` [n_seqs, n] (float32) is added to the
    tokens ``bias_ids`` (int32; ids outside the vocabulary are empty places, the
    last of equal ids counts); tokens whose bit in ``allowed`` (int32 [rows or 1,
    ceil(vocab / 32)]) is 0 become -inf.  ``out`` (logits itself, or memory
    apart from them) receives the result; with ``write`` false only the best tokens are computed."""
    lib = _library()
    torch = _op.torch
    if _op._forward_ad._current_level >= 0:
        _no_tangents(logits, tokens, history, history_lengths, prompt_lengths, repetition, frequency, presence, bias_ids,
                     bias, allowed, out)
    dev = _batch(batch)
    S = batch.n_seqs
    if logits.device != dev:
        _refuse("logits must be on the batch's device")
    ls = _op._matrix(logits, "logits")
    code = _dtype(logits.dtype, "logits")
    rows, V = logits.shape
    batch._check_rows(rows, MAX_ADJUST_ROWS, False)
    if not 1 <= V <= MAX_VOCAB:
        _refuse(f"the vocabulary may have up to {MAX_VOCAB} tokens")
    tp = _array(tokens, "tokens", torch.int32, (rows,), dev) if tokens is not None else 0
    hp = hs = hn = hl = pl = 0
    if history is not None:
        if history_lengths is None:
            _refuse("history needs history_lengths")
        hp, hs, hn = _table(history, "history", torch.int32, S, dev)
        if hn > MAX_HISTORY:
            _refuse(f"a history may have up to {MAX_HISTORY} tokens")
        hl = _array(history_lengths, "history_lengths", torch.int32, (S,), dev)
        if prompt_lengths is not None:
            pl = _array(prompt_lengths, "prompt_lengths", torch.int32, (S,), dev)
    elif history_lengths is not None or prompt_lengths is not None:
        _refuse("history_lengths and prompt_lengths belong to a history")
    if (bias is None) != (bias_ids is None):
        _refuse("bias and bias_ids go together")
    bi = bis = b = bs = nb = 0
    if bias is not None:
        bi, bis, nb = _table(bias_ids, "bias_ids", torch.int32, S, dev)
        b, bs, m = _table(bias, "bias", torch.float32, S, dev)
        if m != nb or nb > MAX_BIAS:
            _refuse(f"bias and bias_ids must have one shape, up to {MAX_BIAS} columns")
    ap = as_ = 0
    if allowed is not None:
        ap, as_, w = _table(allowed, "allowed", torch.int32, 1 if allowed.dim() == 2 and allowed.shape[0] == 1 else rows, dev)
        if w != (V + 31) // 32:
            _refuse(f"allowed must have {(V + 31) // 32} columns")
        if allowed.shape[0] == 1:
            as_ = 0
    best = torch.empty(rows, dtype=torch.int32, device=dev)
    dst, op, os_ = out, 0, 0
    if out is not None:
        if not write:
            _refuse("out needs write=True")
        os_ = _op._matrix(out, "out", dev, rows, V)
        if out.dtype != logits.dtype:
            _refuse("out must have logits' dtype")
        op = out.data_ptr()
    elif write:
        dst, os_ = torch.empty((rows, V), dtype=logits.dtype, device=dev), V
        op = dst.data_ptr()
    args = _pack_adjust(logits.data_ptr(), ls, op, os_, best.data_ptr(), tp, hp, hs, hl, pl,
                        _per_seq(repetition, "repetition", S, dev), _per_seq(frequency, "frequency", S, dev),
                        _per_seq(presence, "presence", S, dev), bi, bis, b, bs, ap, as_, V, hn, nb, code)
    key = (rows, V, code)
    n = batch._sizes.get(key)
    if n is None:
        n = lib.hvd_adjust_workspace(batch._p, args, rows)
        if n == 0:
            raise HvdError(HVD_ERR_ARG, lib.hvd_last_error().decode())
        if len(batch._sizes) >= 256:
            batch._sizes.clear()
        batch._sizes[key] = n
    work = torch.empty(n, dtype=torch.uint8, device=dev)
    _call(dev, lib.hvd_adjust_logits, batch._p, args, rows, work.data_ptr(), n)
    if out is not None:
        _written(out)
    return dst, best
