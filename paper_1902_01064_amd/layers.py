"""Layers of a residual block on all replicas at once, on PyTorch tensors: the calls of include/hop_layers.h.

The rows (samples, tokens) of all groups - workers of a wave, or experts - lie stacked in one matrix, group g's from row_begin[g] up to
row_begin[g + 1] (an int32 tensor on the GPU), and every group has parameters of its own.  A parameter is a tensor [M, ...] with M = G, or with
`index` (a list of G row numbers) a view of more: of an arena of replicas [workers x slots, stride], one row is one version of
one worker, and `arena[:, at:at + n].unflatten(1, (out, in))` is a layer's weights in all of them.  Nothing is copied; gradients are
written the same way, so `out=` can be the N x d tensor that hop_set_grad_source(ctx, HOP_GRAD_EXTERNAL, ...) was given.

Rows are float32 or bfloat16 with contiguous columns; the distance between rows is free.  Calls enqueue kernels on the current
stream and return.  What the library refuses raises HopError, what does not fit together ValueError or TypeError; nothing falls
back to anything else.

Gradients are calls of their own: results carry no history for torch's differentiation.  Where that is enabled, a tensor that requires a
gradient is refused (call under torch.no_grad(), or with detached tensors); what `out=` and its like are given counts as changed in place.
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
# A kernel of a small call takes less time than its launch (4 us), so what is asked of the arguments is asked in the order that lets plain
# ones through with few questions, and devices are compared as numbers.
_raw_stream = torch._C._cuda_getCurrentRawStream
_changed = torch.autograd.graph.increment_version


def _needs_history(name):
    if torch.is_grad_enabled():
        raise ValueError("%s requires a gradient, which would be lost: results have no history (torch.no_grad() or detach() say that none is wanted)" % name)


def _rows(x, name):
    """(type, GPU, distance between rows, rows, columns) of the tensor that a call goes by."""
    try:
        dtype = _TYPES[x.dtype]
    except KeyError:
        raise TypeError("%s: float32 or bfloat16 is needed, got %s" % (name, x.dtype)) from None
    if x.requires_grad:
        _needs_history(name)
    gpu = x.get_device()
    if gpu < 0:
        raise ValueError("%s: a tensor on the GPU is needed" % name)
    if gpu != torch.cuda.current_device():
        raise ValueError("%s is on cuda:%d, the current device is cuda:%d" % (name, gpu, torch.cuda.current_device()))
    shape = x.shape
    if len(shape) != 2:
        raise ValueError("%s: a matrix is needed, got %s" % (name, list(shape)))
    return dtype, gpu, _distance(x, name, shape[0], shape[1]), shape[0], shape[1]


def _distance(t, name, rows, cols):
    ld, step = t.stride()
    if step == 1 and ld >= cols or rows == 0:
        return ld if ld >= cols else cols
    if cols > 1 and step != 1:
        raise ValueError("%s: columns have to be contiguous, got strides %s" % (name, list(t.stride())))
    if rows > 1 and ld < cols:
        raise ValueError("%s: rows overlap, got strides %s" % (name, list(t.stride())))
    return max(ld, cols)


def _ld(t, name, dtype, gpu, rows, cols):
    """Distance between the rows of a matrix that has to be rows x cols."""
    if t.shape != (rows, cols):
        raise ValueError("%s: a matrix [%d, %d] is needed, got %s" % (name, rows, cols, list(t.shape)))
    if t.dtype is not dtype:
        raise TypeError("%s: %s is needed, got %s" % (name, dtype, t.dtype))
    if t.get_device() != gpu:
        raise ValueError("%s: a tensor on cuda:%d is needed" % (name, gpu))
    if t.requires_grad:
        _needs_history(name)
    return _distance(t, name, rows, cols)


def _table(row_begin, gpu):
    """(address, G) of a row table."""
    if row_begin is None:
        return 0, 1
    if row_begin.dtype is not torch.int32 or row_begin.get_device() != gpu or row_begin.dim() != 1 or row_begin.shape[0] < 2 or row_begin.stride(0) != 1:
        raise ValueError("row_begin: a contiguous int32 vector of G + 1 row numbers on cuda:%d is needed" % gpu)
    return row_begin.data_ptr(), row_begin.shape[0] - 1


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


def _vector(t, name, cols, gpu, M=None):
    """(address, distance, M) of a parameter [M, cols] in float32."""
    if t is None:
        return 0, 0, M
    shape = t.shape
    if len(shape) != 2 or shape[1] != cols or t.dtype is not torch.float32 or t.get_device() != gpu or (cols > 1 and t.stride(1) != 1):
        raise ValueError("%s: float32 [groups, %d] with contiguous columns on cuda:%d is needed" % (name, cols, gpu))
    if t.requires_grad:
        _needs_history(name)
    if M is not None and shape[0] != M:
        raise ValueError("%s: %d rows, other parameters have %d" % (name, shape[0], M))
    return t.data_ptr(), t.stride(0), shape[0]


def _weights(w, name, gpu):
    """(distance between groups, distance between rows, shape) of [M, rows, columns]."""
    shape, stride = w.shape, w.stride()
    if len(shape) != 3 or w.get_device() != gpu or (shape[2] > 1 and stride[2] != 1) or (shape[1] > 1 and stride[1] < shape[2]):
        raise ValueError("%s: [groups, rows, columns] with contiguous columns on cuda:%d is needed, got %s with strides %s"
                         % (name, gpu, list(shape), list(stride)))
    if w.requires_grad:
        _needs_history(name)
    return stride[0], max(stride[1], shape[2]), shape


def _result(t, x, name, gpu, rows, cols):
    """(tensor, address, distance) of a result like x."""
    if t is None:
        t = x.new_empty((rows, cols))
        return t, t.data_ptr(), cols
    ld = _ld(t, name, x.dtype, gpu, rows, cols)
    _changed(t)
    return t, t.data_ptr(), ld


def _with_scratch(name, like, gpu, *args):
    """The call, with scratch if it says that it needs some (most do not, and asking each of them first would cost another call)."""
    lib = _lib or load()
    rc = getattr(lib, name)(*args, None, 0, _raw_stream(gpu))
    if rc == hop.HOP_ERR_ARENA_TOO_SMALL:
        need = getattr(lib, name + "_scratch_bytes")(*args)
        s = like.new_empty(need, dtype=torch.uint8)
        rc = getattr(lib, name)(*args, s.data_ptr(), need, _raw_stream(gpu))
    if rc:
        hop._check(rc, name)


def _drop(drop):
    if drop is None:
        return None
    try:
        return _DROP(drop.seed & ((1 << 64) - 1), drop.first_row, drop.worker, drop.iter, drop.site, drop.p)
    except struct.error as e:
        raise ValueError("%s: %s" % (drop, e)) from None


def _at(packed):
    return C.cast(C.c_char_p(packed), C.c_void_p).value if packed is not None else 0


# ------------------------------------------------------------------------------------------- products ----
def product(x, w, row_begin=None, index=None, transposed=False, out=None):
    """y[r] = w_g x[r] for the rows r of group g; w [M, out, in].  transposed: y[r] = w_g^T x[r] - the gradient to x from
    one to y, with the same w."""
    dtype, gpu, ldx, rows, k = _rows(x, "x")
    table, G = _table(row_begin, gpu)
    step, ldw, (M, a, b) = _weights(w, "w", gpu)
    if transposed:
        a, b = b, a
    if w.dtype is not x.dtype or b != k:
        raise ValueError("w: %s [groups, %s] is needed, got %s %s" % (x.dtype, "%d, out" % k if transposed else "out, %d" % k, w.dtype, list(w.shape)))
    idx = _index(index, G, M, "w")
    out, y_at, ldy = _result(out, x, "out", gpu, rows, a)
    args = _PRODUCT(rows, table, G, dtype, x.data_ptr(), ldx, w.data_ptr(), ldw, step, _address(idx), y_at, ldy, k, a,
                    1 if transposed else 0, 0)
    _with_scratch("hop_product", x, gpu, args)
    return out


def product_grad(dy, x, row_begin=None, out=None, index=None):
    """dw_g = sum over the group's rows of dy[r] x[r]^T, in float32: [G, out, in], or into the rows `index` of `out`."""
    dtype, gpu, ldx, rows, k = _rows(x, "x")
    if dy.dim() != 2 or dy.shape[0] != rows:
        raise ValueError("dy: a matrix of x's %d rows is needed, got %s" % (rows, list(dy.shape)))
    n = dy.shape[1]
    lddy = _ld(dy, "dy", x.dtype, gpu, rows, n)
    table, G = _table(row_begin, gpu)
    if out is None:
        if index is not None:
            raise ValueError("index without out")
        out = x.new_empty((G, n, k), dtype=torch.float32)
    elif out.dtype is not torch.float32 or out.shape[1:] != (n, k):
        raise ValueError("out: float32 [groups, %d, %d] is needed, got %s %s" % (n, k, out.dtype, list(out.shape)))
    step, lddw, (M, _, _) = _weights(out, "out", gpu)
    idx = _index(index, G, M, "out")
    _changed(out)
    args = _PRODUCT_GRAD(rows, table, G, dtype, dy.data_ptr(), lddy, x.data_ptr(), ldx, out.data_ptr(), lddw, step, _address(idx), k, n)
    _with_scratch("hop_product_grad", x, gpu, args)
    return out


# -------------------------------------------------------------------------------------------- dropout ----
def dropout(x, drop, out=None):
    """x / (1 - p) where the mask of `drop` keeps it, else 0.  The gradient is dropout(dy, drop)."""
    dtype, gpu, ldx, rows, cols = _rows(x, "x")
    out, y_at, ldy = _result(out, x, "out", gpu, rows, cols)
    hop._check((_lib or load()).hop_dropout(dtype, x.data_ptr(), ldx, y_at, ldy, rows, cols, _drop(drop), _raw_stream(gpu)), "hop_dropout")
    return out


# ------------------------------------------------------------------------------ norms around a block ----
def _residual_args(rows, cols, dtype, like, gpu, b, row_begin, index, norm, post, gate, logits, scale, drop, next_norm, pre, eps):
    """(packed hop_residual_args, what has to live as long, G)."""
    table, G = _table(row_begin, gpu)
    b_at, ldb = (0, 0) if b is None else (b.data_ptr(), _ld(b, "b", like, gpu, rows, cols))
    post_at, post_step, M = _vector(post, "post", cols, gpu)
    pre_at, pre_step, M = _vector(pre, "pre", cols, gpu, M)
    gate_at, gate_step, M = _vector(gate, "gate", cols, gpu, M)
    kind, z_at, ldz = HOP_GATE_NONE if gate is None else HOP_GATE_VECTOR, 0, 0
    if logits is not None:
        if gate is not None:
            raise ValueError("gate and gate_logits: there is one gate")
        kind, z_at, ldz = HOP_GATE_ELEMENT, logits.data_ptr(), _ld(logits, "gate_logits", like, gpu, rows, cols)
    idx = None if M is None else _index(index, G, M, "post, pre, gate")
    packed = _drop(drop)
    try:
        norm, next_norm = _NORMS[norm], _NORMS[next_norm]
    except (KeyError, TypeError):
        raise ValueError("norm: None, 'rms' or 'centred'") from None
    try:
        args = _RESIDUAL(rows, table, G, dtype, cols, b_at, ldb, z_at, ldz, post_at, post_step, pre_at, pre_step, gate_at, gate_step, _address(idx),
                         _at(packed), norm, next_norm, kind, scale, eps, 0)
    except struct.error as e:
        raise ValueError("scale %s, eps %s: %s" % (scale, eps, e)) from None
    return args, (idx, packed), G


def residual(x, b, row_begin=None, index=None, norm="rms", post=None, gate=None, gate_logits=None, scale=1.0, drop=None, next_norm=None, pre=None, eps=1e-5,
             out=None, out_next=None):
    """y = x + scale * dropout(gate * norm(b) * post), h = next_norm(y) * pre: (y, h), h None without next_norm.

    post, pre: [M, cols] float32 or None (1).  The gate is `gate`, [M, cols] float32, as it is; or the logistic function of
    `gate_logits`, a tensor like x; or 1.  norm, next_norm: None, "rms", "centred"."""
    dtype, gpu, ldx, rows, cols = _rows(x, "x")
    if b is None:
        raise ValueError("b: a matrix is needed (norm() is a norm by itself)")
    args, keep, _ = _residual_args(rows, cols, dtype, x.dtype, gpu, b, row_begin, index, norm, post, gate, gate_logits, scale, drop, next_norm, pre, eps)
    if next_norm is None and out_next is not None:
        raise ValueError("out_next without next_norm")
    y, y_at, ldy = _result(out, x, "out", gpu, rows, cols)
    h, h_at, ldh = (None, None, 0) if next_norm is None else _result(out_next, x, "out_next", gpu, rows, cols)
    hop._check((_lib or load()).hop_residual(args, x.data_ptr(), ldx, y_at, ldy, h_at, ldh, _raw_stream(gpu)), "hop_residual")
    del keep
    return y, h


def norm(x, pre=None, row_begin=None, index=None, norm="rms", eps=1e-5, out=None):
    """norm(x) * pre: the norm before a network's first block."""
    dtype, gpu, ldx, rows, cols = _rows(x, "x")
    args, keep, _ = _residual_args(rows, cols, dtype, x.dtype, gpu, None, row_begin, index, None, None, None, None, 1.0, None, norm, pre, eps)
    h, h_at, ldh = _result(out, x, "out", gpu, rows, cols)
    hop._check((_lib or load()).hop_residual(args, x.data_ptr(), ldx, None, 0, h_at, ldh, _raw_stream(gpu)), "hop_residual")
    del keep
    return h


def residual_grad(dy, dh, y, b, row_begin=None, index=None, norm="rms", post=None, gate=None, gate_logits=None, scale=1.0, drop=None,
                  next_norm=None, pre=None, eps=1e-5, dpost=None, dpre=None, dgate=None, grad_index=None, dx=None, db=None, dlogits=None):
    """Gradients of residual() with the same arguments: dy, dh those of its results (one of them may be None), y its result.

    dpost, dpre, dgate: where the parameters' gradients go ([M, cols] float32, written in the rows grad_index), or None for new tensors
    [G, cols].  dx, db, dlogits likewise, like x."""
    like = dy if dy is not None else dh
    if like is None:
        raise ValueError("dy and dh are both None")
    dtype, gpu, ld, rows, cols = _rows(like, "dy" if dy is not None else "dh")
    if dh is not None and (next_norm is None or y is None):
        raise ValueError("dh needs next_norm and residual's result y")
    args, keep, G = _residual_args(rows, cols, dtype, like.dtype, gpu, b, row_begin, index, norm, post, gate, gate_logits, scale, drop, next_norm, pre, eps)
    dy_at, lddy = (0, 0) if dy is None else (dy.data_ptr(), ld)
    dh_at, lddh, y_at, ldy = 0, 0, 0, 0
    if dh is not None:
        dh_at, lddh = dh.data_ptr(), ld if dy is None else _ld(dh, "dh", like.dtype, gpu, rows, cols)
        y_at, ldy = y.data_ptr(), _ld(y, "y", like.dtype, gpu, rows, cols)

    def matrix(t, name, wanted):
        if wanted:
            return _result(t, like, name, gpu, rows, cols)
        if t is not None:
            raise ValueError("%s: there is nothing to differentiate" % name)
        return None, 0, 0

    dx, dx_at, lddx = matrix(dx, "dx", True)
    db, db_at, lddb = matrix(db, "db", b is not None)
    dlogits, dz_at, lddz = matrix(dlogits, "dlogits", gate_logits is not None)
    M, packed = None, []
    grads = [dpost, dpre, dgate]
    params = (post, pre if dh is not None else None, gate)
    if dpost is dpre is dgate is None and grad_index is None:          # new ones: parts of one allocation, nothing to check
        wanted = [i for i in range(3) if params[i] is not None]
        if wanted:
            M = G
            for i, t in zip(wanted, like.new_empty((len(wanted), G, cols), dtype=torch.float32).unbind(0)):
                grads[i] = t
        for t in grads:
            packed += (0, 0) if t is None else (t.data_ptr(), cols)
    else:
        for i, name in enumerate(("dpost", "dpre", "dgate")):
            if params[i] is None and grads[i] is not None:
                raise ValueError("%s: there is nothing to differentiate" % name)
            if params[i] is not None and grads[i] is None:
                if grad_index is not None:
                    raise ValueError("grad_index without %s" % name)
                grads[i] = like.new_empty((G, cols), dtype=torch.float32)
            at, step, M = _vector(grads[i], name, cols, gpu, M)
            if grads[i] is not None:
                _changed(grads[i])
            packed += (at, step)
    idx = None if M is None else _index(grad_index, G, M, "dpost, dpre, dgate")
    out = _GRADS(dy_at, lddy, dh_at, lddh, y_at, ldy, dx_at, lddx, db_at, lddb, dz_at, lddz, *packed, _address(idx))
    lib = _lib or load()
    need = 0 if M is None else lib.hop_residual_grad_scratch_bytes(args, out)
    scratch = like.new_empty(need, dtype=torch.uint8) if need else None
    hop._check(lib.hop_residual_grad(args, out, scratch.data_ptr() if need else None, need, _raw_stream(gpu)), "hop_residual_grad")
    del keep
    return ResidualGrads(dx, db, *grads, dlogits)


def norm_grad(dh, x, pre=None, row_begin=None, index=None, norm="rms", eps=1e-5, dy=None, dpre=None, grad_index=None, dx=None):
    """Gradients (dx, dpre) of norm(); dy: one that reaches x by another way, added to dx."""
    g = residual_grad(dy, dh, x, None, row_begin=row_begin, index=index, norm=None, next_norm=norm, pre=pre, eps=eps, dpre=dpre,
                      grad_index=grad_index, dx=dx)
    return g.dx, g.dpre
