"""Refusals of the operators on rows in 8 bits: every bad argument is named by a
status before anything is launched (no GPU is touched)."""
import ctypes
import os

import pytest
import torch  # noqa: F401  (loads the HIP runtime libgcn links against)

from paper_2010_12635_amd import gcn as G

pytestmark = pytest.mark.skipif(not os.path.exists(G.LIB_PATH), reason="libgcn.so not built")

INVALID, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 6
NAN = float("nan")
WIDE = G.Q8_MAX_WIDTH + 16


def quantize(n=10, f=20, prec=1, h=0x1000, ld=24, kind=0, q=0x2000, ldq=32, s=0x3000, ov=None):
    return G.lib().gcn_quantize(n, f, prec, h, ld, kind, q, ldq, s, ov, None)


def dequantize(n=10, f=20, prec=1, h=0x1000, ld=24, kind=0, q=0x2000, ldq=32, s=0x3000, ov=None):
    return G.lib().gcn_dequantize(n, f, kind, q, ldq, s, prec, h, ld, ov, None)


def weights(f=20, n=10, prec=1, h=0x1000, ld=16, q=0x2000, ldq=32, s=0x3000, ws=0x4000, ov=None):
    return G.lib().gcn_quantize_weights(f, n, prec, h, ld, q, ldq, s, ws, ov, None)


def product(n=10, f=20, fo=7, kind=1, q=0x1000, ldq=32, s=0x2000, w=0x3000, ldw=32, wsc=0x4000, wsum=0x5000, prec=1,
            out=0x6000, ld=8, ov=None):
    return G.lib().gcn_transform_q8(n, f, fo, kind, q, ldq, s, w, ldw, wsc, wsum, prec, out, ld, ov, None)


def backward(n=10, f=20, fo=7, prec=1, kind=1, q=0x1000, ldq=32, s=0x2000, w=0x3000, ldw=8, g=0x4000, ldg=8, act=1,
             p=0.5, dw=0x5000, dz=0x6000, ldz=24, db=0x7000, ov=None, ws=0x8000, wb=1 << 30):
    return G.lib().gcn_transform_bwd_q8(n, f, fo, prec, kind, q, ldq, s, w, ldw, g, ldg, act, p, dw, dz, ldz, db, ov, ws,
                                        wb, None)


def layer(n=10, f=20, fo=7, prec=1, kind=1, q=0x1000, ldq=32, s=0x2000, w=0x3000, g=0x4000, act=1, p=0.5, dw=0x5000,
          dz=0x6000, db=0x7000, dzt=0x9000, dbt=None, ov=None, ws=0x8000, wb=1 << 30, ident=0, ldi=24, ldo=8, adj=True):
    a = G.GcnAdj()
    a.n, a.nnz, a.index, a.value_prec = n, 30, G.GCN_I32, prec
    a.rowptr, a.colidx, a.values, a.dinv = 0x100000, 0x200000, 0x300000, 0x400000
    L = G.GcnLayer(f, fo, ldi, ldo, 0, 0.0, 0, ident)
    return G.lib().gcn_layer_bwd_q8(ctypes.byref(a) if adj else None, ctypes.byref(L), prec, kind, q, ldq, s, w, dzt, act,
                                    p, dw, dbt, dz, db, g, ov, ws, wb, None)


ALL = [quantize, dequantize, product, backward, layer]


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("args,status", [
    (dict(prec=3), INVALID), (dict(prec=-1), INVALID), (dict(kind=2), INVALID), (dict(kind=-1), INVALID),
    (dict(n=0), SHAPE), (dict(n=-5), SHAPE), (dict(f=0), SHAPE), (dict(ldq=16), SHAPE), (dict(ldq=40), ALIGN),
    (dict(n=1 << 31), UNSUPPORTED), (dict(q=None), INVALID), (dict(s=None), INVALID), (dict(q=0x1008), ALIGN),
    (dict(s=0x2004), ALIGN)])
def test_codes(call, args, status):
    assert call(**args) == status


@pytest.mark.parametrize("call", [quantize, dequantize])
@pytest.mark.parametrize("args,status", [
    (dict(h=None), INVALID), (dict(h=0x1004), ALIGN), (dict(ld=16), SHAPE), (dict(ld=28), ALIGN),
    (dict(f=WIDE, ld=WIDE, ldq=WIDE), UNSUPPORTED)])
def test_rows(call, args, status):
    assert call(**args) == status


@pytest.mark.parametrize("args,status", [
    (dict(prec=5), INVALID), (dict(f=0), SHAPE), (dict(n=0), SHAPE), (dict(ld=8), SHAPE), (dict(ld=20), ALIGN),
    (dict(ldq=16), SHAPE), (dict(ldq=40), ALIGN), (dict(f=WIDE, ldq=WIDE), UNSUPPORTED),
    (dict(n=WIDE, ld=WIDE), UNSUPPORTED), (dict(h=None), INVALID), (dict(q=None), INVALID), (dict(s=None), INVALID),
    (dict(ws=None), INVALID), (dict(h=0x1002), ALIGN), (dict(q=0x2008), ALIGN), (dict(s=0x3004), ALIGN),
    (dict(ws=0x4004), ALIGN)])
def test_weights(args, status):
    assert weights(**args) == status


@pytest.mark.parametrize("args,status", [
    (dict(fo=0), SHAPE), (dict(ldw=16), SHAPE), (dict(ldw=40), ALIGN), (dict(ld=0), SHAPE), (dict(ld=12), ALIGN),
    (dict(f=WIDE, ldq=WIDE, ldw=WIDE), UNSUPPORTED), (dict(fo=WIDE, ld=WIDE), UNSUPPORTED), (dict(w=None), INVALID),
    (dict(wsc=None), INVALID), (dict(wsum=None), INVALID), (dict(out=None), INVALID), (dict(w=0x3008), ALIGN),
    (dict(wsc=0x4004), ALIGN), (dict(wsum=0x5004), ALIGN), (dict(kind=0, wsum=0x5004), ALIGN), (dict(out=0x6004), ALIGN)])
def test_product(args, status):
    assert product(**args) == status


@pytest.mark.parametrize("call", [backward, layer])
@pytest.mark.parametrize("args,status", [
    (dict(fo=0), SHAPE), (dict(w=None), INVALID), (dict(g=None), INVALID), (dict(dw=None), INVALID),
    (dict(dz=None), INVALID), (dict(act=2), INVALID), (dict(p=1.0), INVALID), (dict(p=-0.5), INVALID),
    (dict(p=NAN), INVALID), (dict(kind=0), UNSUPPORTED), (dict(w=0x3004), ALIGN), (dict(g=0x4008), ALIGN),
    (dict(dw=0x5004), ALIGN), (dict(dz=0x6004), ALIGN), (dict(db=0x7004), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(wb=0), WORKSPACE), (dict(ws=0x8004), ALIGN)])
def test_backward(call, args, status):
    assert call(**args) == status


@pytest.mark.parametrize("args,status", [
    (dict(ldw=0), SHAPE), (dict(ldw=12), ALIGN), (dict(ldg=0), SHAPE), (dict(ldg=12), ALIGN), (dict(ldz=16), SHAPE),
    (dict(ldz=28), ALIGN), (dict(f=WIDE, ldq=WIDE, ldz=WIDE), UNSUPPORTED),
    (dict(fo=WIDE, ldw=WIDE, ldg=WIDE), UNSUPPORTED),
    (dict(ldw=1 << 60), UNSUPPORTED),
    (dict(f=65536, fo=16384, ldq=65536, ldz=65536, ldw=16384, ldg=16384), UNSUPPORTED)])
def test_backward_shapes(args, status):
    assert backward(**args) == status


@pytest.mark.parametrize("args,status", [
    (dict(adj=False), INVALID), (dict(ident=1, f=10, ldi=16), INVALID), (dict(dzt=None), INVALID),
    (dict(dzt=0x9008), ALIGN), (dict(dbt=0x9004), ALIGN), (dict(ldi=20), ALIGN), (dict(ldi=16), SHAPE),
    (dict(ldo=4), SHAPE)])
def test_layer(args, status):
    assert layer(**args) == status


def test_workspace_sizes():
    size = G.gcn_transform_bwd_q8_workspace_size
    assert size(1, 1, 1, 0) > 0 and size(1 << 21, 128, 64, 1) > size(1, 128, 64, 1) > 0
    for bad, status in (((0, 7, 7, 1), SHAPE), ((7, 0, 7, 1), SHAPE), ((7, 7, 0, 1), SHAPE), ((7, 7, 7, 3), INVALID),
                        ((7, WIDE, 7, 1), UNSUPPORTED), ((1 << 31, 7, 7, 1), UNSUPPORTED),
                        ((7, 65536, 65536, 1), UNSUPPORTED)):
        with pytest.raises(G.GcnError) as e:
            size(*bad)
        assert e.value.status == status
    a = G.GcnAdj()
    a.n, a.nnz, a.value_prec, a.rowptr, a.colidx, a.dinv = 100, 300, 1, 0x1000, 0x2000, 0x3000
    small = G.gcn_layer_bwd_q8_workspace_size(a, G.GcnLayer(16, 7, 16, 8, 0, 0.0, 1, 0), 1)
    assert 0 < small < G.gcn_layer_bwd_q8_workspace_size(a, G.GcnLayer(160, 70, 160, 72, 0, 0.0, 1, 0), 1)
    with pytest.raises(G.GcnError) as e:
        G.gcn_layer_bwd_q8_workspace_size(a, G.GcnLayer(100, 7, 104, 8, 0, 0.0, 1, 1), 1)
    assert e.value.status == INVALID
