"""What the layers' C ABI refuses (host code only: every call here is turned down before a kernel is launched)."""
import os
import re
import struct

import pytest

from paper_1902_01064_amd import hop, layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                                   # an address that nothing reads
INF, NAN = float("inf"), float("nan")


def test_library_exports_what_the_header_declares():
    text = open(os.path.join(ROOT, "include", "hop_layers.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(hop_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(layers.EXPORTS)
    for n in names:
        assert hasattr(layers.load(), n)


def ints(*v):
    a = layers.array("i", v)
    return a.buffer_info()[0], a


def product(**over):
    f = dict(rows=4, table=A, G=2, dtype=0, x=A, ldx=8, w=A, ldw=8, w_stride=64, w_index=0, y=A, ldy=8, k=8, n=8, t=0)
    f.update(over)
    return layers._PRODUCT(f["rows"], f["table"], f["G"], f["dtype"], f["x"], f["ldx"], f["w"], f["ldw"], f["w_stride"], f["w_index"],
                           f["y"], f["ldy"], f["k"], f["n"], f["t"], 0)


BAD = hop.HOP_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [
    dict(rows=-1), dict(rows=1 << 31), dict(G=0), dict(G=layers.HOP_MAX_GROUPS + 1), dict(dtype=2), dict(dtype=-1), dict(table=0), dict(table=A + 2),
    dict(x=0), dict(x=A + 2), dict(ldx=7), dict(w=0), dict(ldw=7), dict(y=0), dict(ldy=7), dict(k=0), dict(n=0), dict(k=(1 << 21) + 1), dict(n=(1 << 21) + 1),
    dict(k=9), dict(n=9), dict(dtype=1, x=A + 1), dict(t=1, n=9), dict(ldx=1 << 41), dict(w_stride=1 << 41)])
def test_product(over):
    assert layers.load().hop_product(product(**over), A, 1 << 30, 0) == BAD


def test_product_indexes():
    at, keep = ints(0, -1)
    assert layers.load().hop_product(product(w_index=at), A, 1 << 30, 0) == BAD
    many = layers.array("i", range(layers.HOP_MAX_INDEXED + 1))
    assert layers.load().hop_product(product(G=len(many), w_index=many.buffer_info()[0]), A, 1 << 30, 0) == BAD
    assert layers.load().hop_product(None, A, 1 << 30, 0) == BAD
    assert layers.load().hop_product(product(rows=0, x=0, y=0), None, 0, 0) == 0          # nothing to do


def grad(**over):
    f = dict(rows=4, table=A, G=2, dtype=0, dy=A, lddy=8, x=A, ldx=8, dw=A, lddw=8, dw_stride=64, index=0, k=8, n=8)
    f.update(over)
    return layers._PRODUCT_GRAD(f["rows"], f["table"], f["G"], f["dtype"], f["dy"], f["lddy"], f["x"], f["ldx"], f["dw"], f["lddw"],
                                f["dw_stride"], f["index"], f["k"], f["n"])


@pytest.mark.parametrize("over", [dict(rows=-1), dict(G=0), dict(dtype=5), dict(table=0), dict(dy=0), dict(lddy=7), dict(x=0), dict(ldx=7),
                                  dict(dw=0), dict(dw=A + 2), dict(lddw=7), dict(k=0), dict(n=0), dict(rows=0, dw=0)])
def test_product_grad(over):
    assert layers.load().hop_product_grad(grad(**over), A, 1 << 30, 0) == BAD


def test_product_grad_two_groups_into_one_place():
    at, keep = ints(3, 3)
    assert layers.load().hop_product_grad(grad(index=at), A, 1 << 30, 0) == BAD


def drop(p=0.5, first=0):
    return struct.pack("@Qqiiif", 1, first, 0, 0, 0, p)


@pytest.mark.parametrize("args", [
    (2, A, 8, A, 8, 4, 8, drop()), (0, 0, 8, A, 8, 4, 8, drop()), (0, A, 7, A, 8, 4, 8, drop()), (0, A, 8, 0, 8, 4, 8, drop()),
    (0, A, 8, A + 64, 7, 4, 8, drop()), (0, A, 8, A, 9, 4, 8, drop()), (0, A, 8, A, 8, -1, 8, drop()), (0, A, 8, A, 8, 4, 0, drop()),
    (0, A, 8, A, 8, 4, 8, None), (0, A, 8, A, 8, 4, 8, drop(-0.1)), (0, A, 8, A, 8, 4, 8, drop(1.5)), (0, A, 8, A, 8, 4, 8, drop(NAN)),
    (0, A, 8, A, 8, 4, 8, drop(0.5, -1)), (0, A, 8, A, 8, 4, 8, drop(0.5, (1 << 63) - 1)), (1, A + 1, 8, A, 8, 4, 8, drop())])
def test_dropout(args):
    assert layers.load().hop_dropout(*args, 0) == BAD


def residual(**over):
    f = dict(rows=4, table=A, G=2, dtype=0, cols=8, b=A, ldb=8, z=0, ldz=0, post=A, post_s=8, pre=A, pre_s=8, gate=0, gate_s=0, index=0, drop=0,
             norm=1, next=1, kind=0, scale=1.0, eps=1e-5)
    f.update(over)
    return layers._RESIDUAL(f["rows"], f["table"], f["G"], f["dtype"], f["cols"], f["b"], f["ldb"], f["z"], f["ldz"], f["post"], f["post_s"],
                            f["pre"], f["pre_s"], f["gate"], f["gate_s"], f["index"], f["drop"], f["norm"], f["next"], f["kind"], f["scale"],
                            f["eps"], 0)


ARGS = [dict(rows=-1), dict(table=0), dict(G=0), dict(dtype=3), dict(cols=0), dict(cols=layers.HOP_MAX_NORM_COLS + 1), dict(ldb=7), dict(b=A + 2),
        dict(norm=3), dict(norm=-1), dict(next=3), dict(kind=3), dict(kind=1), dict(kind=2), dict(kind=1, gate=A, z=A, ldz=8), dict(kind=0, gate=A),
        dict(kind=0, z=A, ldz=8), dict(kind=2, z=A, ldz=7), dict(kind=2, z=A, ldz=8, gate=A), dict(scale=INF), dict(scale=NAN), dict(eps=-1.0),
        dict(eps=NAN), dict(eps=INF), dict(b=0), dict(next=0), dict(b=0, post=0, norm=0, next=0, pre=0), dict(post=A + 1), dict(pre=A + 2)]


@pytest.mark.parametrize("over", ARGS)
def test_residual(over):
    assert layers.load().hop_residual(residual(**over), A, 8, A, 8, A, 8, 0) == BAD


@pytest.mark.parametrize("at", [(0, 8, A, 8, A, 8), (A, 7, A, 8, A, 8), (A, 8, 0, 8, A, 8), (A, 8, A, 7, A, 8), (A, 8, A, 8, 0, 8), (A, 8, A, 8, A, 7),
                                (A + 1, 8, A, 8, A, 8)])
def test_residual_tensors(at):
    assert layers.load().hop_residual(residual(), *at, 0) == BAD
    assert layers.load().hop_residual(residual(next=0, pre=0), A, 8, A, 8, A, 8, 0) == BAD      # h for no norm


def grads(**over):
    f = dict(dy=A, lddy=8, dh=A, lddh=8, y=A, ldy=8, dx=A, lddx=8, db=A, lddb=8, dz=0, lddz=0, dpost=A, dpost_s=8, dpre=A, dpre_s=8, dgate=0,
             dgate_s=0, index=0)
    f.update(over)
    return layers._GRADS(*f.values())


GRADS = [dict(lddy=7), dict(lddh=7), dict(ldy=7), dict(lddx=7), dict(lddb=7), dict(y=0), dict(dy=0, dh=0), dict(dz=A, lddz=8), dict(dgate=A),
         dict(dpost=A + 2), dict(dx=A + 2)]


@pytest.mark.parametrize("over", GRADS)
def test_residual_grad(over):
    assert layers.load().hop_residual_grad(residual(), grads(**over), A, 1 << 30, 0) == BAD


@pytest.mark.parametrize("over", ARGS)
def test_residual_grad_arguments(over):
    assert layers.load().hop_residual_grad(residual(**over), grads(), A, 1 << 30, 0) == BAD
    assert layers.load().hop_residual_grad_scratch_bytes(residual(**over), grads()) == 0


def test_residual_grad_scratch():
    lib = layers.load()
    need = lib.hop_residual_grad_scratch_bytes(residual(), grads())
    assert need > 0
    assert lib.hop_residual_grad(residual(), grads(), A, need - 1, 0) == hop.HOP_ERR_ARENA_TOO_SMALL
    assert lib.hop_residual_grad(residual(), grads(), None, need, 0) == BAD
    assert lib.hop_residual_grad(residual(), grads(), A + 8, need, 0) == BAD
    assert lib.hop_residual_grad_scratch_bytes(residual(), grads(dpost=0, dpre=0)) == 0
    at, keep = ints(5, 5)
    assert lib.hop_residual_grad(residual(), grads(index=at), A, 1 << 30, 0) == BAD
    assert lib.hop_residual_grad(residual(b=0, post=0, norm=0), grads(dpost=0), A, 1 << 30, 0) == BAD       # db of no block
