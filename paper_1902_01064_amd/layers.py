"""Layers of a residual block on all replicas at once, on PyTorch tensors: the calls of include/hop_layers.h.

The rows (samples, tokens) of all groups - workers of a wave, or experts - lie stacked in one matrix, group g's from row_begin[g] up to
row_begin[g + 1] (an int32 tensor on the GPU), and every group has parameters of its own.  A parameter is a tensor [M, ...] with M = G, or with
`index` (a list of G row numbers) a view of more: of an arena of replicas [workers x slots, stride], one row is one version of
one worker, and `arena[:, at:at + n].unflatten(1, (out, in))` is a layer's weights in all of them.  Nothing is copied; gradients are
written the same way, so `out=` can be the N x d tensor that hop_set_grad_source(ctx, HOP_GRAD_EXTERNAL, ...) was given.

Rows are float32 or bfloat16 with contiguous columns; the distance between rows is free.  Calls enqueue kernels on the current
stream and return.  What the library refuses raises HopError, what does not fit together ValueError or TypeError; nothing falls
back to anything else.
"""
import collections
import ctypes as C
import struct
from array import array

import torch

from . import hop

HOP_F32, HOP_BF16 = 0, 1
HOP_NORM_NONE, HOP_NORM_RMS, HOP_NORM_CENTRED = 0, 1, 2
HOP_GATE_NONE, HOP_GATE_VECTOR, HOP_GATE_ELEMENT = 0, 1, 2
HOP_MAX_GROUPS, HOP_MAX_INDEXED, HOP_MAX_NORM_COLS = 4096, 256, 32768

EXPORTS = ["hop_product_scratch_bytes", "hop_product", "hop_product_grad_scratch_bytes", "hop_product_grad", "hop_dropout",
           "hop_residual", "hop_residual_grad_scratch_bytes", "hop_residual_grad"]

_TYPES = {torch.float32: HOP_F32, torch.bfloat16: HOP_BF16}
_NORMS = {None: HOP_NORM_NONE, "rms": HOP_NORM_RMS, "centred": HOP_NORM_CENTRED}

# the structures of hop_layers.h as bytes (setting ctypes fields one by one takes several times as long)
_GROUPS = "qPii"
_PRODUCT = struct.Struct("@" + _GROUPS + "PqPqqPPqqqii").pack
_PRODUCT_GRAD = struct.Struct("@" + _GROUPS + "PqPqPqqPqq").pack
_DROP = struct.Struct("@Qqiiif").pack
_RESIDUAL = struct.Struct("@" + _GROUPS + "qPqPqPqPqPqPPiiiffi").pack
_GRADS = struct.Struct("@" + "Pq" * 9 + "P").pack

#: A dropout: probability and what its mask is drawn from (see hop_layers.h).  first_row: row number of the first row.
Drop = collections.namedtuple("Drop", "p seed worker iter site first_row", defaults=(0, 0, 0, 0))

#: What residual_grad returns; None where there is nothing to differentiate.
ResidualGrads = collections.namedtuple("ResidualGrads", "dx db dpost dpre dgate dlogits")

_lib = None


def load():
    """libhop.so with the signatures of hop_layers.h."""
    global _lib
    if _lib is None:
        lib = hop.load()
        vp, i32, i64, size = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        args = C.c_char_p                         # packed structures
        for name, res, types in (("hop_product_scratch_bytes", size, [args]), ("hop_product", C.c_int, [args, vp, size, vp]),
                                 ("hop_product_grad_scratch_bytes", size, [args]), ("hop_product_grad", C.c_int, [args, vp, size, vp]),
                                 ("hop_dropout", C.c_int, [i32, vp, i64, vp, i64, i64, i64, args, vp]),
                                 ("hop_residual", C.c_int, [args, vp, i64, vp, i64, vp, i64, vp]),
                                 ("hop_residual_grad_scratch_bytes", size, [args, args]),
                                 ("hop_residual_grad", C.c_int, [args, args, vp, size, vp])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, types
        _lib = lib
    return _lib


# ------------------------------------------------------------------------------------------ arguments ----
def _ld(t, name, dtype, shape=None):
    """Distance between the rows of a matrix."""
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError("%s: a matrix %s is needed, got %s" % (name, "" if shape is None else list(shape), list(t.shape)))
    if t.dtype != dtype:
        raise TypeError("%s: %s is needed, got %s" % (name, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s: a tensor on the GPU is needed" % name)
    rows, cols = t.shape
    ld, step = t.stride()
    if rows == 0:
        return cols
    if cols > 1 and step != 1:
        raise ValueError("%s: columns have to be contiguous, got strides %s" % (name, list(t.stride())))
    if rows == 1:
        return max(ld, cols)
    if ld < cols:
        raise ValueError("%s: rows overlap, got strides %s" % (name, list(t.stride())))
    return ld


def _type(t, name):
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise TypeError("%s: float32 or bfloat16 is needed, got %s" % (name, t.dtype)) from None


def _table(row_begin, device):
    """(address, G) of a row table."""
    if row_begin is None:
        return 0, 1
    if row_begin.dtype != torch.int32 or row_begin.dim() != 1 or row_begin.numel() < 2 or not row_begin.is_contiguous() or row_begin.device != device:
        raise ValueError("row_begin: a contiguous int32 vector of G + 1 row numbers on %s is needed" % device)
    return row_begin.data_ptr(), row_begin.numel() - 1


def _index(index, G, M, name):
    """An index list as an array (kept alive by the caller), or None."""
    if index is None:
        if M != G:
            raise ValueError("%s: %d parameters for %d groups, and no index" % (name, M, G))
        return None
    if len(index) != G or (G and not (0 <= min(index) and max(index) < M)):
        raise ValueError("index: %d numbers below %d are needed, got %s" % (G, M, list(index)[:8]))
    return array("i", index)


def _address(a):
    return 0 if a is None else a.buffer_info()[0]


def _vector(t, name, cols, device, M=None):
    """(address, distance, M) of a parameter [M, cols] in float32."""
    if t is None:
        return 0, 0, M
    if t.dim() != 2 or t.shape[1] != cols or t.dtype != torch.float32 or t.device != device or (cols > 1 and t.stride(1) != 1):
        raise ValueError("%s: float32 [groups, %d] with contiguous columns on %s is needed" % (name, cols, device))
    if M is not None and t.shape[0] != M:
        raise ValueError("%s: %d rows, other parameters have %d" % (name, t.shape[0], M))
    return t.data_ptr(), t.stride(0), t.shape[0]


def _weights(w, name, device):
    if w.dim() != 3 or w.device != device or (w.shape[2] > 1 and w.stride(2) != 1) or (w.shape[1] > 1 and w.stride(1) < w.shape[2]):
        raise ValueError("%s: [groups, rows, columns] with contiguous columns on %s is needed, got %s with strides %s"
                         % (name, device, list(w.shape), list(w.stride())))
    return max(w.stride(1), w.shape[2])


def _stream(t):
    return torch.cuda.current_stream(t.device).cuda_stream


def _on(t):
    """Kernels run on the tensors' GPU, whichever is the current one."""
    if torch.cuda.current_device() != t.device.index:
        raise ValueError("tensors are on %s, the current device is cuda:%d" % (t.device, torch.cuda.current_device()))


def _scratch(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _drop(drop):
    return None if drop is None else _DROP(drop.seed & ((1 << 64) - 1), drop.first_row, drop.worker, drop.iter, drop.site, drop.p)


def _at(packed):
    return C.cast(C.c_char_p(packed), C.c_void_p).value if packed is not None else 0


# ------------------------------------------------------------------------------------------- products ----
def product(x, w, row_begin=None, index=None, transposed=False, out=None):
    """y[r] = w_g x[r] for the rows r of group g; w [M, out, in].  transposed: y[r] = w_g^T x[r] - the gradient to x from
    one to y, with the same w."""
    lib, dtype = load(), _type(x, "x")
    ldx = _ld(x, "x", x.dtype)
    rows, k = x.shape
    table, G = _table(row_begin, x.device)
    ldw = _weights(w, "w", x.device)
    if w.dtype != x.dtype or w.shape[1 if transposed else 2] != k:
        raise ValueError("w: %s [groups, %s] is needed, got %s %s" % (x.dtype, "%d, out" % k if transposed else "out, %d" % k, w.dtype, list(w.shape)))
    n = w.shape[2 if transposed else 1]
    idx = _index(index, G, w.shape[0], "w")
    if out is None:
        out = torch.empty((rows, n), dtype=x.dtype, device=x.device)
        ldy = n
    else:
        ldy = _ld(out, "out", x.dtype, (rows, n))
    _on(x)
    a = _PRODUCT(rows, table, G, dtype, x.data_ptr(), ldx, w.data_ptr(), ldw, w.stride(0), _address(idx), out.data_ptr(), ldy, k, n,
                 1 if transposed else 0, 0)
    need = lib.hop_product_scratch_bytes(a)
    s = _scratch(need, x.device)
    hop._check(lib.hop_product(a, s.data_ptr() if need else None, need, _stream(x)), "hop_product")
    return out


def product_grad(dy, x, row_begin=None, out=None, index=None):
    """dw_g = sum over the group's rows of dy[r] x[r]^T, in float32: [G, out, in], or into the rows `index` of `out`."""
    lib, dtype = load(), _type(x, "x")
    lddy, ldx = _ld(dy, "dy", x.dtype), _ld(x, "x", x.dtype)
    if dy.shape[0] != x.shape[0]:
        raise ValueError("dy has %d rows, x %d" % (dy.shape[0], x.shape[0]))
    (rows, n), k = dy.shape, x.shape[1]
    table, G = _table(row_begin, x.device)
    if out is None:
        if index is not None:
            raise ValueError("index without out")
        out = torch.empty((G, n, k), dtype=torch.float32, device=x.device)
    elif out.dtype != torch.float32 or out.shape[1:] != (n, k):
        raise ValueError("out: float32 [groups, %d, %d] is needed, got %s %s" % (n, k, out.dtype, list(out.shape)))
    lddw = _weights(out, "out", x.device)
    idx = _index(index, G, out.shape[0], "out")
    _on(x)
    a = _PRODUCT_GRAD(rows, table, G, dtype, dy.data_ptr(), lddy, x.data_ptr(), ldx, out.data_ptr(), lddw, out.stride(0), _address(idx), k, n)
    need = lib.hop_product_grad_scratch_bytes(a)
    s = _scratch(need, x.device)
    hop._check(lib.hop_product_grad(a, s.data_ptr() if need else None, need, _stream(x)), "hop_product_grad")
    return out


# -------------------------------------------------------------------------------------------- dropout ----
def dropout(x, drop, out=None):
    """x / (1 - p) where the mask of `drop` keeps it, else 0.  The gradient is dropout(dy, drop)."""
    dtype = _type(x, "x")
    ldx = _ld(x, "x", x.dtype)
    rows, cols = x.shape
    if out is None:
        out = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        ldy = cols
    else:
        ldy = _ld(out, "out", x.dtype, x.shape)
    _on(x)
    hop._check(load().hop_dropout(dtype, x.data_ptr(), ldx, out.data_ptr(), ldy, rows, cols, _drop(drop), _stream(x)), "hop_dropout")
    return out


# ------------------------------------------------------------------------------ norms around a block ----
def _residual_args(rows, cols, dtype, b, row_begin, index, norm, post, gate, logits, scale, drop, next_norm, pre, eps, device, torch_type):
    """(packed hop_residual_args, what has to live as long, G)."""
    table, G = _table(row_begin, device)
    ldb = 0 if b is None else _ld(b, "b", torch_type, (rows, cols))
    post_at, post_step, M = _vector(post, "post", cols, device)
    pre_at, pre_step, M = _vector(pre, "pre", cols, device, M)
    gate_at, gate_step, M = _vector(gate, "gate", cols, device, M)
    kind, z_at, ldz = HOP_GATE_NONE if gate is None else HOP_GATE_VECTOR, 0, 0
    if logits is not None:
        if gate is not None:
            raise ValueError("gate and gate_logits: there is one gate")
        kind, z_at, ldz = HOP_GATE_ELEMENT, logits.data_ptr(), _ld(logits, "gate_logits", torch_type, (rows, cols))
    idx = None if M is None else _index(index, G, M, "post, pre, gate")
    packed = _drop(drop)
    try:
        norm, next_norm = _NORMS[norm], _NORMS[next_norm]
    except (KeyError, TypeError):
        raise ValueError("norm: None, 'rms' or 'centred'") from None
    a = _RESIDUAL(rows, table, G, dtype, cols, 0 if b is None else b.data_ptr(), ldb, z_at, ldz, post_at, post_step, pre_at, pre_step,
                  gate_at, gate_step, _address(idx), _at(packed), norm, next_norm, kind, scale, eps, 0)
    return a, (idx, packed), G


def residual(x, b, row_begin=None, index=None, norm="rms", post=None, gate=None, gate_logits=None, scale=1.0, drop=None, next_norm=None, pre=None, eps=1e-5,
             out=None, out_next=None):
    """y = x + scale * dropout(gate * norm(b) * post), h = next_norm(y) * pre: (y, h), h None without next_norm.

    post, pre: [M, cols] float32 or None (1).  The gate is `gate`, [M, cols] float32, as it is; or the logistic function of
    `gate_logits`, a tensor like x; or 1.  norm, next_norm: None, "rms", "centred"."""
    dtype = _type(x, "x")
    ldx = _ld(x, "x", x.dtype)
    rows, cols = x.shape
    if b is None:
        raise ValueError("b: a matrix is needed (norm() is a norm by itself)")
    a, keep, _ = _residual_args(rows, cols, dtype, b, row_begin, index, norm, post, gate, gate_logits, scale, drop, next_norm, pre, eps, x.device, x.dtype)
    y = torch.empty((rows, cols), dtype=x.dtype, device=x.device) if out is None else out
    ldy = _ld(y, "out", x.dtype, x.shape)
    h, ldh = None, 0
    if next_norm is not None:
        h = torch.empty((rows, cols), dtype=x.dtype, device=x.device) if out_next is None else out_next
        ldh = _ld(h, "out_next", x.dtype, x.shape)
    _on(x)
    hop._check(load().hop_residual(a, x.data_ptr(), ldx, y.data_ptr(), ldy, None if h is None else h.data_ptr(), ldh, _stream(x)), "hop_residual")
    del keep
    return y, h


def norm(x, pre=None, row_begin=None, index=None, norm="rms", eps=1e-5, out=None):
    """norm(x) * pre: the norm before a network's first block."""
    dtype = _type(x, "x")
    ldx = _ld(x, "x", x.dtype)
    a, keep, _ = _residual_args(*x.shape, dtype, None, row_begin, index, None, None, None, None, 1.0, None, norm, pre, eps, x.device, x.dtype)
    h = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    ldh = _ld(h, "out", x.dtype, x.shape)
    _on(x)
    hop._check(load().hop_residual(a, x.data_ptr(), ldx, None, 0, h.data_ptr(), ldh, _stream(x)), "hop_residual")
    del keep
    return h


def residual_grad(dy, dh, y, b, row_begin=None, index=None, norm="rms", post=None, gate=None, gate_logits=None, scale=1.0, drop=None,
                  next_norm=None, pre=None, eps=1e-5, dpost=None, dpre=None, dgate=None, grad_index=None, dx=None, db=None, dlogits=None):
    """Gradients of residual() with the same arguments: dy, dh those of its results (one of them may be None), y its result.

    dpost, dpre, dgate: where the parameters' gradients go ([M, cols] float32, written in the rows grad_index), or None for new tensors
    [G, cols].  dx, db, dlogits likewise, like x."""
    first = dy if dy is not None else dh
    if first is None:
        raise ValueError("dy and dh are both None")
    dtype, like, device = _type(first, "dy"), first.dtype, first.device
    rows, cols = shape = first.shape
    if dh is not None and (next_norm is None or y is None):
        raise ValueError("dh needs next_norm and residual's result y")
    a, keep, G = _residual_args(rows, cols, dtype, b, row_begin, index, norm, post, gate, gate_logits, scale, drop, next_norm, pre, eps, device, like)
    lddy = 0 if dy is None else _ld(dy, "dy", like)
    lddh = 0 if dh is None else _ld(dh, "dh", like, shape)
    ldy = 0 if dh is None else _ld(y, "y", like, shape)

    def matrix(t, name, wanted):
        if not wanted:
            if t is not None:
                raise ValueError("%s: there is nothing to differentiate" % name)
            return None, 0, 0
        if t is None:
            t = torch.empty(shape, dtype=like, device=device)
        return t, t.data_ptr(), _ld(t, name, like, shape)

    dx, dx_at, lddx = matrix(dx, "dx", True)
    db, db_at, lddb = matrix(db, "db", b is not None)
    dlogits, dz_at, lddz = matrix(dlogits, "dlogits", gate_logits is not None)
    M, packed = None, []
    grads = [dpost, dpre, dgate]
    for i, (name, p) in enumerate((("dpost", post), ("dpre", pre if dh is not None else None), ("dgate", gate))):
        if p is None and grads[i] is not None:
            raise ValueError("%s: there is nothing to differentiate" % name)
        if p is not None and grads[i] is None:
            if grad_index is not None:
                raise ValueError("grad_index without %s" % name)
            grads[i] = torch.empty((G, cols), dtype=torch.float32, device=device)
        at, step, M = _vector(grads[i], name, cols, device, M)
        packed += [at, step]
    idx = None if M is None else _index(grad_index, G, M, "dpost, dpre, dgate")
    _on(first)
    out = _GRADS(0 if dy is None else dy.data_ptr(), lddy, 0 if dh is None else dh.data_ptr(), lddh, 0 if dh is None else y.data_ptr(), ldy,
                 dx_at, lddx, db_at, lddb, dz_at, lddz, *packed, _address(idx))
    lib = load()
    need = lib.hop_residual_grad_scratch_bytes(a, out)
    s = _scratch(need, device)
    hop._check(lib.hop_residual_grad(a, out, s.data_ptr() if need else None, need, _stream(first)), "hop_residual_grad")
    del keep
    return ResidualGrads(dx, db, *grads, dlogits)


def norm_grad(dh, x, pre=None, row_begin=None, index=None, norm="rms", eps=1e-5, dy=None, dpre=None, grad_index=None, dx=None):
    """Gradients (dx, dpre) of norm(); dy: one that reaches x by another way, added to dx."""
    g = residual_grad(dy, dh, x, None, row_begin=row_begin, index=index, norm=None, next_norm=norm, pre=pre, eps=eps, dpre=dpre,
                      grad_index=grad_index, dx=dx)
    return g.dx, g.dpre
