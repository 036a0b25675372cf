"""Attention over the sequences of all replicas at once, and the norm and rotation of its queries and keys, on PyTorch tensors: the calls of
include/hop_attention.h.

Rows are tokens, as in `layers`: matrices in float32 or bfloat16 with contiguous columns and any distance between rows, so that queries, keys and
values may be columns of the matrix that one product wrote (qkv[:, :n] and so on), and a gradient's three parts columns of another.  A head is
a run of columns; query head h belongs to key head h // (q_heads / k_heads).  Sequences lie packed: tables of S + 1 row numbers (int32, on the GPU)
say which rows are whose, and a sequence may have none.

Streams, errors, scratch, indexes of parameters and what happens to tensors that require a gradient are as in `layers`.
"""
import ctypes as C
import struct

import torch

from . import hop, layers
from .layers import _address, _changed, _distance, _index, _ld, _raw_stream, _result, _rows, _vector

HOP_MAX_HEAD_COLS, HOP_MAX_HEADS = 128, 1024

EXPORTS = ["hop_rotate", "hop_rotate_grad_scratch_bytes", "hop_rotate_grad", "hop_attention_scratch_bytes", "hop_attention",
           "hop_attention_grad_scratch_bytes", "hop_attention_grad"]

# the structures of hop_attention.h as bytes
_ROTATE = struct.Struct("@" + layers._GROUPS + "PPiiiiiiPqPqPdfi").pack
_ROTATE_GRADS = struct.Struct("@" + "Pq" * 5 + "P").pack
_ATTENTION = struct.Struct("@qqPPii" + "Pq" * 3 + "iiiifi").pack
_ATTENTION_GRADS = struct.Struct("@PqPqPPqPqPq").pack

_lib = None


def load():
    """libhop.so with the signatures of hop_attention.h."""
    global _lib
    if _lib is None:
        lib = layers.load()
        vp, i64, size = C.c_void_p, C.c_int64, C.c_size_t
        args = C.c_char_p                         # packed structures
        for name, res, types in (("hop_rotate", C.c_int, [args, vp, i64, vp, i64, vp]), ("hop_rotate_grad_scratch_bytes", size, [args, args]),
                                 ("hop_rotate_grad", C.c_int, [args, args, vp, size, vp]), ("hop_attention_scratch_bytes", size, [args]),
                                 ("hop_attention", C.c_int, [args, vp, i64, vp, vp, size, vp]), ("hop_attention_grad_scratch_bytes", size, [args, args]),
                                 ("hop_attention_grad", C.c_int, [args, args, vp, size, vp])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, types
        _lib = lib
    return _lib


def _sequences(begin, name, gpu):
    """(address, S) of a table of sequences."""
    if begin is None:
        return 0, 1
    if begin.dtype is not torch.int32 or begin.get_device() != gpu or begin.dim() != 1 or begin.shape[0] < 2 or begin.stride(0) != 1:
        raise ValueError("%s: a contiguous int32 vector of S + 1 row numbers on cuda:%d is needed" % (name, gpu))
    return begin.data_ptr(), begin.shape[0] - 1


def _columns(name, cols, heads):
    if heads < 1 or cols % heads:
        raise ValueError("%s: %d columns are not those of %d heads" % (name, cols, heads))
    return cols // heads


# ------------------------------------------------------------------------------------- norm and rotation ----
def _rotate_args(rows, cols, dtype, gpu, q_heads, k_heads, q_weight, k_weight, row_begin, index, positions, seq_begin, rotary, adjacent, base, norm, eps):
    """(packed hop_rotate_args, what has to live as long, G, columns of a head)."""
    head = _columns("x", cols, q_heads + k_heads)
    table, G = layers._table(row_begin, gpu)
    q_at, q_step, M = _vector(q_weight, "q_weight", head, gpu)
    k_at, k_step, M = _vector(k_weight, "k_weight", head, gpu, M)
    idx = None if M is None else _index(index, G, M, "q_weight, k_weight")
    at = 0
    if positions is not None:
        if positions.dtype is not torch.int32 or positions.get_device() != gpu or positions.shape != (rows,) or (rows > 1 and positions.stride(0) != 1):
            raise ValueError("positions: a contiguous int32 vector of %d numbers on cuda:%d is needed" % (rows, gpu))
        at = positions.data_ptr()
    seq, S = _sequences(seq_begin, "seq_begin", gpu)
    if norm not in layers._NORMS:
        raise ValueError("norm: None, 'rms' or 'centred'")
    try:
        args = _ROTATE(rows, table, G, dtype, at, seq, S, q_heads, k_heads, head, head if rotary is None else rotary, 1 if adjacent else 0, q_at, q_step, k_at, k_step,
                       _address(idx), base, eps, layers._NORMS[norm])
    except struct.error as e:
        raise ValueError("heads %s and %s, rotary %s, base %s, eps %s: %s" % (q_heads, k_heads, rotary, base, eps, e)) from None
    return args, idx, G, head


def rotate(x, q_heads, k_heads, q_weight=None, k_weight=None, row_begin=None, index=None, positions=None, seq_begin=None, rotary=None, adjacent=False,
           base=10000.0, norm="rms", eps=1e-5, out=None):
    """The heads of queries and keys (x: rows x (q_heads + k_heads) heads, the queries' first), each normed, times the weight of its kind and the row's
    group, its first `rotary` columns (None: all) turned by the row's position: in pairs of columns half of `rotary` apart, or `adjacent` ones.

    q_weight, k_weight: [M, columns of a head] float32 or None (1).  positions: int32 of every row; None: the row's number in its sequence
    of seq_begin.  norm: "rms", "centred" or None.  `out` may be x (whose gradient then needs a copy of x)."""
    dtype, gpu, ldx, rows, cols = _rows(x, "x")
    args, keep, _, _ = _rotate_args(rows, cols, dtype, gpu, q_heads, k_heads, q_weight, k_weight, row_begin, index, positions, seq_begin, rotary, adjacent,
                                    base, norm, eps)
    out, y_at, ldy = _result(out, x, "out", gpu, rows, cols)
    hop._check((_lib or load()).hop_rotate(args, x.data_ptr(), ldx, y_at, ldy, _raw_stream(gpu)), "hop_rotate")
    del keep
    return out


def rotate_grad(dy, x, q_heads, k_heads, q_weight=None, k_weight=None, row_begin=None, index=None, positions=None, seq_begin=None, rotary=None, adjacent=False,
                base=10000.0, norm="rms", eps=1e-5, dq_weight=None, dk_weight=None, grad_index=None, dx=None):
    """Gradients (dx, dq_weight, dk_weight) of rotate() with the same arguments; x as rotate got it.

    dq_weight, dk_weight: where the weights' gradients go ([M, columns] float32, written in the rows grad_index), or None for new tensors [G, columns];
    None is returned for a weight that there is none of.  dx may be dy."""
    dtype, gpu, lddy, rows, cols = _rows(dy, "dy")
    ldx = _ld(x, "x", dy.dtype, gpu, rows, cols)
    args, keep, G, head = _rotate_args(rows, cols, dtype, gpu, q_heads, k_heads, q_weight, k_weight, row_begin, index, positions, seq_begin, rotary, adjacent,
                                       base, norm, eps)
    dx, dx_at, lddx = _result(dx, dy, "dx", gpu, rows, cols)
    M, packed, grads = None, [], [dq_weight, dk_weight]
    for i, (name, weight) in enumerate((("dq_weight", q_weight), ("dk_weight", k_weight))):
        if weight is None and grads[i] is not None:
            raise ValueError("%s: there is nothing to differentiate" % name)
        if weight is not None and grads[i] is None:
            if grad_index is not None:
                raise ValueError("grad_index without %s" % name)
            grads[i] = dy.new_empty((G, head), dtype=torch.float32)
        at, step, M = _vector(grads[i], name, head, gpu, M)
        if grads[i] is not None:
            _changed(grads[i])
        packed += (at, step)
    idx = None if M is None else _index(grad_index, G, M, "dq_weight, dk_weight")
    g = _ROTATE_GRADS(dy.data_ptr(), lddy, x.data_ptr(), ldx, dx_at, lddx, *packed, _address(idx))
    lib = _lib or load()
    need = 0 if M is None else lib.hop_rotate_grad_scratch_bytes(args, g)
    scratch = dy.new_empty(need, dtype=torch.uint8) if need else None
    hop._check(lib.hop_rotate_grad(args, g, scratch.data_ptr() if need else None, need, _raw_stream(gpu)), "hop_rotate_grad")
    del keep
    return dx, grads[0], grads[1]


# --------------------------------------------------------------------------------------------- attention ----
def _attention_args(q, k, v, q_heads, k_heads, q_begin, k_begin, causal, scale):
    """(packed hop_attention_args, GPU, query rows, key rows, columns of q, columns of k)."""
    dtype, gpu, ldq, q_rows, wide = _rows(q, "q")
    head = _columns("q", wide, q_heads)
    if k.dim() != 2:
        raise ValueError("k: a matrix is needed, got %s" % list(k.shape))
    k_rows, narrow = k.shape[0], k_heads * head
    ldk, ldv = _ld(k, "k", q.dtype, gpu, k_rows, narrow), _ld(v, "v", q.dtype, gpu, k_rows, narrow)
    q_at, S = _sequences(q_begin, "q_begin", gpu)
    if k_begin is None and q_begin is not None:
        if k_rows != q_rows:
            raise ValueError("k_begin: a table is needed where there are %d keys for %d queries" % (k_rows, q_rows))
        k_at = q_at
    else:
        k_at, n = _sequences(k_begin, "k_begin", gpu)
        if n != S:
            raise ValueError("k_begin: %d sequences, q_begin has %d" % (n, S))
    try:
        args = _ATTENTION(q_rows, k_rows, q_at, k_at, S, dtype, q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, q_heads, k_heads, head, 1 if causal else 0,
                          head ** -0.5 if scale is None else scale, 0)
    except struct.error as e:
        raise ValueError("heads %s and %s, scale %s: %s" % (q_heads, k_heads, scale, e)) from None
    return args, gpu, q_rows, k_rows, wide, narrow


def _lse(t, like, gpu, heads, rows, name):
    if t.shape != (heads, rows) or t.dtype is not torch.float32 or t.get_device() != gpu or not t.is_contiguous():
        raise ValueError("%s: a contiguous float32 matrix [%d, %d] on cuda:%d is needed" % (name, heads, rows, gpu))
    if t.requires_grad:
        layers._needs_history(name)
    return t.data_ptr()


def attention(q, k, v, q_heads, k_heads, q_begin=None, k_begin=None, causal=True, scale=None, out=None, out_lse=None):
    """o = softmax(scale q k^T) v head by head within each sequence, and the logarithms of the softmaxes' sums [q_heads, rows] in float32: (o, lse).

    q: rows x q_heads heads; k, v: rows x k_heads heads.  q_begin, k_begin: the sequences' rows among the queries and the keys (one sequence without;
    k_begin None: the same as q_begin).  causal: the queries are the last rows of their sequence, each sees the keys up to itself; so with one
    query row to a sequence this is the step that writes the next token.  scale: None for 1 / sqrt(columns of a head)."""
    args, gpu, rows, _, wide, _ = _attention_args(q, k, v, q_heads, k_heads, q_begin, k_begin, causal, scale)
    out, o_at, ldo = _result(out, q, "out", gpu, rows, wide)
    if out_lse is None:
        out_lse = q.new_empty((q_heads, rows), dtype=torch.float32)
        lse_at = out_lse.data_ptr()
    else:
        lse_at = _lse(out_lse, q, gpu, q_heads, rows, "out_lse")
        _changed(out_lse)
    lib = _lib or load()
    need = lib.hop_attention_scratch_bytes(args)
    scratch = q.new_empty(need, dtype=torch.uint8) if need else None
    hop._check(lib.hop_attention(args, o_at, ldo, lse_at, scratch.data_ptr() if need else None, need, _raw_stream(gpu)), "hop_attention")
    return out, out_lse


def attention_grad(do, o, lse, q, k, v, q_heads, k_heads, q_begin=None, k_begin=None, causal=True, scale=None, dq=None, dk=None, dv=None):
    """Gradients (dq, dk, dv) of attention() with the same arguments; do the gradient of its o, o and lse what it returned."""
    args, gpu, q_rows, k_rows, wide, narrow = _attention_args(q, k, v, q_heads, k_heads, q_begin, k_begin, causal, scale)
    lddo, ldo = _ld(do, "do", q.dtype, gpu, q_rows, wide), _ld(o, "o", q.dtype, gpu, q_rows, wide)
    lse_at = _lse(lse, q, gpu, q_heads, q_rows, "lse")
    dq, dq_at, lddq = _result(dq, q, "dq", gpu, q_rows, wide)
    dk, dk_at, lddk = _result(dk, q, "dk", gpu, k_rows, narrow)
    dv, dv_at, lddv = _result(dv, q, "dv", gpu, k_rows, narrow)
    g = _ATTENTION_GRADS(do.data_ptr(), lddo, o.data_ptr(), ldo, lse_at, dq_at, lddq, dk_at, lddk, dv_at, lddv)
    lib = _lib or load()
    need = lib.hop_attention_grad_scratch_bytes(args, g)
    scratch = q.new_empty(need, dtype=torch.uint8) if need else None
    hop._check(lib.hop_attention_grad(args, g, scratch.data_ptr() if need else None, need, _raw_stream(gpu)), "hop_attention_grad")
    return dq, dk, dv
